"""A teacher's entries that lie close together against the temperature: bounds from the differences of a row's entries, not from their quotients."""
import numpy as np
import pytest
import torch

from paper_2602_05145_amd import binding as B
from tests.gpu_util import stream, sync
from tests.loss_util import CODE, DEV, HALF, STEP, TDT, assert_within, gen, logits, padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 5001, 200001])
@pytest.mark.parametrize("tau,spread", [(1.0, 2.0), (1e-3, 2e-3), (1e-5, 2e-5), (1e-6, 5e-6), (1.0, 0.0)])
def test_entries_close_together(dtype, vocab, tau, spread):
    """The student is flat (log q = -log vocab to the last step), so that the loss is the teacher's entropy term and the gradient at its columns -tau p.
    p: an exact difference, three roundings of a number of its size d, the exponential, a sum of k terms beside it: 3 d + 24 half steps; a logarithm and
    the differences of numbers up to d + log vocab: 16 half steps of those."""
    rows, k, tau = 20, 9, float(np.float32(tau))
    z = torch.zeros((rows, padded(vocab)), device=DEV, dtype=TDT[dtype])
    ids = torch.stack([torch.randperm(vocab, device=DEV, generator=gen(r))[:k] for r in range(rows)]).to(torch.int32)
    t = 7.0 + spread * torch.rand((rows, k), device=DEV, generator=gen(1)) if spread else torch.full((rows, k), 3e38, device=DEV)
    t[3:6, ::2] -= 1000.0
    mask, lse, loss = torch.ones(rows, dtype=torch.uint8, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    dz = torch.empty_like(z)
    d = (t.double() - t.double().amax(1, keepdim=True)) / tau
    p = torch.softmax(d, 1)
    log_p = d - torch.logsumexp(d, 1, keepdim=True)
    log_v = float(np.log(vocab))
    want = tau * tau * torch.where(p > 0, p * (log_p + log_v), 0.0).sum(1)
    p_rel = (3 * d.abs() + 24) * HALF
    tol = tau * tau * torch.where(p > 1.2e-38, p * (p_rel * (1 + (log_p + log_v).abs()) + 16 * HALF * (log_p.abs() + log_v)), p * log_p.abs()).sum(1)
    tol = 1.01 * tol + tau * tau * (vocab / 256 + 64) * HALF
    at = tau * (1.0 / vocab - p)
    at_tol = 1.01 * tau * (p * p_rel + (vocab / 256 + 80) * HALF / vocab) + 1e-37
    for train in (False, True):
        if train:
            B.tide_distill_train(rows, vocab, z, dz, z.shape[1], k, ids, t, None, tau, mask, lse, loss, CODE[dtype], stream())
        else:
            B.tide_distill_eval(rows, vocab, z, z.shape[1], k, ids, t, None, tau, mask, lse, loss, CODE[dtype], stream())
        sync()
        assert_within(loss, want, tol, ("loss", train))
    assert_within(dz.gather(1, ids.long()), at, at_tol + STEP[dtype] * (at.abs() + at_tol), "dz")
