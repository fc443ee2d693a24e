"""tide_lm_ce_fwd / tide_lm_ce_bwd on logits that are large, infinite or not numbers, and on vocabularies at the limit."""
import math

import pytest
import torch

from paper_2602_05145_amd import binding as B
from tests.gpu_util import stream, sync
from tests.loss_util import CODE, DEV, HALF, STEP, TDT, assert_within, gen

pytestmark = pytest.mark.gpu


def head(y, w, tokens, want_dw=True):
    """(lse, loss, dy, dw) of a head whose rows all count."""
    (rows, d), vocab = y.shape, w.shape[0]
    code = CODE["bf16" if y.dtype == torch.bfloat16 else "fp32"]
    ws = torch.empty(B.tide_lm_ce_workspace_bytes(rows, vocab, d, code), dtype=torch.uint8, device=DEV).fill_(0xFF)
    mask = torch.ones(rows, dtype=torch.uint8, device=DEV)
    lse, loss = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    dy, dw = torch.empty_like(y), torch.empty_like(w) if want_dw else None
    B.tide_lm_ce_fwd(rows, vocab, d, y, w, tokens, mask, lse, loss, code, ws, ws.numel(), stream())
    B.tide_lm_ce_bwd(rows, vocab, d, y, w, tokens, mask, lse, None, 1.0, dy, dw, code, code, ws, ws.numel(), stream())
    sync()
    return lse, loss, dy, dw


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("scale", [2.0 ** 8, 2.0 ** 20, 2.0 ** 30, 2.0 ** 33, 2.0 ** 60, 2.0 ** 110])
@pytest.mark.parametrize("vocab,rows", [(200, 3), (1000, 40), (5003, 300)])
def test_large_logits(dtype, scale, vocab, rows):
    """Logits without a rounding (one term each, of few bits), of which every row has one that is the largest by scale / 64 or more: log S is 0 to the last
    bit of fp32, lse is that logit, the loss its difference to the label's, and dz is 1 there and -1 at the label (0 where they are one)."""
    d = 8
    g = gen(vocab)
    top = torch.randperm(vocab, device=DEV, generator=g)[:d]
    w = torch.zeros((vocab, d), device=DEV)
    w[:, 1] = torch.randint(0, 62, (vocab,), device=DEV, generator=g) / 64.0
    w[top, 1] = 1.0 + torch.arange(d, device=DEV) / 64.0
    y = torch.zeros((rows, d), device=DEV)
    y[:, 1] = scale
    y[1::3, 1] = -scale                                 # the smallest weight is the largest logit then
    w[:, 1] += 0.5
    w[top[0], 1] = 0.25
    z = y.double() @ w.double().T
    best = z.argmax(1)
    tokens = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
    tokens[::2] = best[::2]
    lse, loss, dy, dw = head(y.to(TDT[dtype]), w.to(TDT[dtype]), tokens.to(torch.int32))
    at = torch.arange(rows, device=DEV)
    gap = z[at, best] - z.scatter(1, best[:, None], -math.inf).amax(1)
    assert float(gap.min()) >= scale / 64
    # what the other logits leave of a probability: vocab exp(-gap); the lse that the backward call gets is rounded
    rest = vocab * torch.exp(-gap)
    assert_within(lse, z[at, best], HALF * z[at, best].abs() + rest + 1e-6, "lse")
    diff = z[at, best] - z[at, tokens]
    assert_within(loss, diff, HALF * diff + rest + 1e-6, "loss")
    dz = torch.zeros_like(z)
    dz[at, best] += 1.0
    dz[at, tokens] -= 1.0
    off = torch.where(tokens == best, 4 * HALF + rest, 4 * HALF + rest + STEP[dtype])    # of each of the one or two that are not nothing
    want = dz @ w.double()
    assert_within(dy, want, 1.01 * (2 * off + rest)[:, None] * w.double().abs().max() + STEP[dtype] * want.abs(), "dy")
    want = dz.T @ y.double()
    off_sum = (off + rest).max() * rows * scale
    assert_within(dw, want, 1.01 * off_sum + (rows + 8) * HALF * (dz.abs().T @ y.double().abs()) + STEP[dtype] * (want.abs() + off_sum), "dw")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [5, 300, 2100])      # tiles of 128, and taller ones
def test_a_logit_that_is_no_number_among_infinite_ones(dtype, rows):
    """256 columns whose logits are -inf but for one NaN, in any of their quarters: the row's log-sum-exp and loss are NaN, whatever the other columns hold;
    without the NaN they are those of the other columns."""
    vocab, d, inf = 1200, 64, math.inf
    for bad in (None, 256, 300, 350, 400, 511):
        g = gen(rows)
        y, w = torch.zeros((rows, d), device=DEV), torch.zeros((vocab, d), device=DEV)
        y[:, 0], y[:, 1], y[:, 2:] = 1.0, 0.5, torch.randn((rows, d - 2), device=DEV, generator=g)
        w[:, 2:] = 0.1 * torch.randn((vocab, d - 2), device=DEV, generator=g)
        w[256:512, 0] = -inf
        if bad is not None:
            w[bad, 1] = inf
        y, w = y.to(TDT[dtype]), w.to(TDT[dtype])
        tokens = torch.randint(0, 256, (rows,), device=DEV, generator=g).to(torch.int32)
        code, mask = CODE[dtype], torch.ones(rows, dtype=torch.uint8, device=DEV)
        ws = torch.empty(B.tide_lm_ce_workspace_bytes(rows, vocab, d, code), dtype=torch.uint8, device=DEV).fill_(0xFF)
        lse, loss = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        B.tide_lm_ce_fwd(rows, vocab, d, y, w, tokens, mask, lse, loss, code, ws, ws.numel(), stream())
        sync()
        if bad is not None:
            assert bool(lse.isnan().all()) and bool(loss.isnan().all()), bad
            continue
        left = torch.cat([w[:256], w[512:]]).double()
        z = y.double() @ left.T
        want = torch.logsumexp(z, 1)
        tol = (d + 2) * HALF * float((y.double().abs() @ left.abs().T).max()) + (vocab / 256 + 64 + 3 * math.log(vocab) + 4) * HALF + 8 * HALF * (math.log(vocab) + 16)
        assert_within(lse, want, tol, "lse")
        assert_within(loss, want - z.gather(1, tokens.long()[:, None])[:, 0], 2 * tol, "loss")


def dz_off(dz, step, lse_tol, ez):
    """An entry of dz is off by its own rounding and, the probability, by what lse and the logits are off; beside 1 by two half steps more."""
    return (step + 2 * lse_tol + 2 * ez + 16 * HALF) * dz.abs() + 2 * HALF * (dz.abs() > 0.5)


@pytest.mark.parametrize("dtype,rows", [("bf16", 1), ("bf16", 5), ("fp32", 4), ("fp32", 6)])
@pytest.mark.parametrize("vocab", [2 ** 21 - 1, 2 ** 21 - 8, 2 ** 21 - 64, 2 ** 21 - 256])
def test_vocabularies_at_the_limit(dtype, rows, vocab):
    """Row lengths of 2^21 are more than the bf16 products take: the pieces stay below.  dz has one large entry per row, at the label, next to probabilities
    of 1 / vocab: the references in 64 bits."""
    d = 8
    g = gen(vocab % 1000 + rows)
    y = torch.randn((rows, d), device=DEV, generator=g).to(TDT[dtype])
    w = torch.randn((vocab, d), device=DEV, generator=g).to(TDT[dtype])
    tokens = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
    tokens[0] = vocab - 1
    lse, loss, dy, dw = head(y, w, tokens.to(torch.int32))
    step, w64 = STEP[dtype], w.double()
    want_dw, dw_tol, want_dy = *torch.zeros((2, vocab, d), dtype=torch.float64, device=DEV), torch.empty((rows, d), dtype=torch.float64, device=DEV)
    for r in range(rows):
        products = w64 * y[r].double()
        z = products.sum(1)
        want = torch.logsumexp(z, 0)
        ez = (d + 2) * HALF * float(products.abs().sum(1).max())
        tol = ez + (vocab / 256 + 64 + 3 * math.log(vocab) + 4) * HALF + 8 * HALF * (math.log(vocab) + 16)
        assert abs(float(lse[r]) - float(want)) <= tol and abs(float(loss[r]) - float(want - z[tokens[r]])) <= 2 * tol, r
        dz = torch.exp(z - want)
        dz[tokens[r]] -= 1.0
        want_dy[r] = (dz[:, None] * w64).sum(0)
        want_dw += dz[:, None] * y[r].double()
        dw_tol += (dz_off(dz, step, tol, ez) + (rows + 8) * HALF * dz.abs())[:, None] * y[r].double().abs()
        off = dz_off(dz, step, tol, ez)
        dy_tol = ((off + (vocab / 32 + 8) * HALF * dz.abs())[:, None] * w64.abs()).sum(0)
        assert bool(((dy[r].double() - want_dy[r]).abs() <= dy_tol + step * (want_dy[r].abs() + dy_tol)).all()), r
    assert bool(((dw.double() - want_dw).abs() <= dw_tol + step * (want_dw.abs() + dw_tol)).all())


@pytest.mark.parametrize("dtype,d", [("bf16", 2 ** 21 - 8), ("bf16", 2 ** 21 - 64), ("fp32", 2 ** 21 - 1), ("fp32", 2 ** 21 - 4)])
def test_widths_at_the_limit(dtype, d):
    rows, vocab = 3, 16
    g = gen(d % 1000)
    y = torch.randn((rows, d), device=DEV, generator=g).to(TDT[dtype])
    w = (torch.randn((vocab, d), device=DEV, generator=g) / 1024.0).to(TDT[dtype])
    tokens = torch.tensor([3, 0, 15], device=DEV)
    lse, loss, dy, dw = head(y, w, tokens.to(torch.int32))
    y64, w64, step = y.double(), w.double(), STEP[dtype]
    products = y64[:, None, :] * w64[None]
    z, ez = products.sum(2), (d + 2) * HALF * products.abs().sum(2).max()
    want = torch.logsumexp(z, 1)
    tol = float(ez) + 100 * HALF * 16
    assert_within(lse, want, tol, "lse")
    assert_within(loss, want - z.gather(1, tokens[:, None])[:, 0], 2 * tol, "loss")
    # (all of a logit's roundings at their worst leave its probability open; at random, 2^17 sums in a row of numbers below 8 make 363 x 8 half steps, 1.8e-4)
    dz = torch.exp(z - want[:, None])
    dz[torch.arange(rows, device=DEV), tokens] -= 1.0
    for got, exact in ((dy, (dz[:, :, None] * w64[None]).sum(1)), (dw, (dz[:, :, None] * y64[:, None, :]).sum(0))):
        assert float((got.double() - exact).norm() / exact.norm()) < step + 2 * 363 * 8 * HALF
