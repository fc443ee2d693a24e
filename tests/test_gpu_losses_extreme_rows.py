"""The losses on rows whose logits are large against their temperature: every row is held to bounds made from that row alone, and from
differences to its largest value, so that a masked column or a neighbour with other numbers widens nothing."""
import math

import numpy as np
import pytest
import torch

from paper_2602_05145_amd import binding as B
from tests.gpu_util import stream, sync
from tests.loss_util import CODE, DEV, HALF, STEP, TDT, assert_within, gen, logits, padded
from tests.test_gpu_topk import _orders

pytestmark = pytest.mark.gpu
FLOAT_MAX = 3.4028235e38


def as_float(tau):
    """The temperature that reaches the library."""
    return float(np.float32(tau))


def statistics(z, tau):
    """Per row in 64 bits: largest value m, log of S = sum exp((z - m) / tau), and what fp32 may be off: of S relative, of log S, of m / tau + log S.
    S: up to n / 256 + 64 additions follow each other (256 threads or more share a row).  A term exp(-x) comes from a difference rounded once, times a
    factor rounded twice: 3 x half steps, weighted with itself at most 3 log n of them (the mean of x under the softmax is below its entropy); the
    instruction and a last factor add 4.  log S: log n at most, good to 4 half steps, after S's error.  The sum: m / tau is rounded once, the
    rounding of a shift (which is no larger than half a step of m / tau) may stand in S, and the result is rounded."""
    z = z.double()
    n = z.shape[1]
    m = z.amax(1)
    x = torch.where(z == m[:, None], 0.0, (z - m[:, None]) / tau)      # (-inf everywhere: no softmax)
    log_s = torch.log(torch.exp(x).sum(1))
    s_rel = (n / 256 + 64 + 3 * math.log(n) + 4) * HALF
    log_tol = s_rel + 4 * HALF * (math.log(n) + 1)
    return m, x, log_s, s_rel, log_tol, m / tau + log_s, log_tol + HALF * (3 * (m / tau).abs() + math.log(n))


def large_rows(vocab, dtype, seed=1):
    """Rows of finite logits on all scales; equal values, close values, and a few columns far above masked ones."""
    z = torch.full((10, padded(vocab, 8)), float("nan"), device=DEV, dtype=TDT[dtype])
    r = 3.0 * torch.randn((10, vocab), device=DEV, generator=gen(seed))
    low = torch.finfo(TDT[dtype]).min
    z[0, :vocab] = -1e9
    z[1, :vocab] = (1e10 + 1500.0 * r[1]).to(TDT[dtype])
    z[2, :vocab] = -1e20
    z[3, :vocab] = r[3].to(TDT[dtype])
    z[4, :vocab] = -1e9
    z[4, 2:vocab:7] = r[4, 2::7].to(TDT[dtype])
    z[5, :vocab] = low
    z[6, :vocab] = (1e6 + r[6]).to(TDT[dtype])
    z[7, :vocab] = -3.1e10
    z[7, vocab - 1] = -3.0e10
    z[8, :vocab] = (7.4e8 + 100.0 * r[8]).to(TDT[dtype])               # times 1 / ln 2 just around 2^30
    z[9, :vocab] = (20.0 + torch.randint(0, 5, (vocab,), device=DEV, generator=gen(seed)).float() * 2.0 ** -19).to(TDT[dtype])
    return z


TAUS = [1.0, 0.3, 1e-3, 1e-6, 50.0, 1e6]
SIZES = [300, 4096, 33001, 128256, 200001]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tau", TAUS)
@pytest.mark.parametrize("rows", [10, 200, 600])        # each number of threads that a row may have
@pytest.mark.parametrize("vocab", [300, 33001])
def test_top_logits(dtype, tau, rows, vocab):
    z = large_rows(vocab, dtype).repeat(rows // 10, 1)
    k, tau = 20, as_float(tau)
    ids, values, lse = torch.empty((rows, k), dtype=torch.int32, device=DEV), torch.empty((rows, k), device=DEV), torch.empty(rows, device=DEV)
    B.tide_topk_logits(rows, vocab, z, z.shape[1], k, tau, ids, values, lse, CODE[dtype], stream())
    sync()
    want_v, want_i = torch.sort(z[:, :vocab].float(), dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), want_i[:, :k]) and torch.equal(values, want_v[:, :k])
    _, _, _, _, _, want, tol = statistics(z[:, :vocab], tau)
    finite = want.abs() < FLOAT_MAX                                       # (the type's lowest value over a small temperature has no fp32 number)
    assert_within(lse[finite], want[finite], tol[finite], "lse")
    assert bool((lse[~finite] == -math.inf).all())


def distill(z, vocab, ids, t, tlse, tau, train):
    rows, ldz = z.shape
    dtype = "bf16" if z.dtype == torch.bfloat16 else "fp32"
    mask = torch.ones(rows, dtype=torch.uint8, device=DEV)
    lse, loss = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    dz = torch.full_like(z, -7.0) if train else None
    if train:
        B.tide_distill_train(rows, vocab, z, dz, ldz, ids.shape[1], ids, t, tlse, tau, mask, lse, loss, CODE[dtype], stream())
    else:
        B.tide_distill_eval(rows, vocab, z, ldz, ids.shape[1], ids, t, tlse, tau, mask, lse, loss, CODE[dtype], stream())
    sync()
    return lse, loss, dz


def check_distill(z, vocab, ids, t, tau, tlse=None):
    """Bounds beside those of statistics(): a teacher's p_j from its difference to the row's largest entry, |d| / tau = a: three roundings of a number of
    size a, the exponential and the sum of k terms beside it (2 a + 24 half steps); with tlse from a quotient and its difference to tlse, each rounded,
    whose sizes are |t| / tau and |tlse|.  Loss: log p_j and log q_j, each from a difference (three roundings) and a logarithm; 16 additions."""
    tau = as_float(tau)
    dtype = "bf16" if z.dtype == torch.bfloat16 else "fp32"
    m, x, log_s, s_rel, log_tol, lse, lse_tol = statistics(z[:, :vocab], tau)
    at_id = x.gather(1, ids.long())
    d = (t.double() - t.double().amax(1, keepdim=True)) / tau
    if tlse is None:
        log_p = d - torch.logsumexp(d, 1, keepdim=True)
        p_rel = (3 * d.abs() + 24) * HALF
    else:
        log_p = t.double() / tau - tlse.double()[:, None]
        p_rel = (4 * (t.double() / tau).abs() + 3 * tlse.double().abs()[:, None] + 24) * HALF
    p = torch.exp(log_p)
    log_q = at_id - log_s[:, None]
    far = torch.where(p > 0, (log_p - log_q).abs(), 0.0)
    term = p_rel * (1 + far) + HALF * (3 * at_id.abs() + 16 * (log_p.abs() + log_q.abs()) + 4 * math.log(ids.shape[1])) + log_tol
    loss = tau * tau * torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1)
    # (a p below the least normal number may be taken for nothing)
    loss_tol = 1.01 * tau * tau * torch.where(p > 1.2e-38, p * term, p * far).sum(1) + tau * tau * 1e-36
    mass, mass_rel = p.sum(1, keepdim=True), (p * p_rel).sum(1, keepdim=True) / p.sum(1, keepdim=True) + 8 * HALF
    q = torch.exp(x - log_s[:, None])
    q_rel = (4 * x.abs().clamp(max=200.0) + 16) * HALF + s_rel
    at = torch.zeros_like(q).scatter_add_(1, ids.long(), p)
    at_tol = torch.zeros_like(q).scatter_add_(1, ids.long(), p * (p_rel + 130 * HALF))
    dz = tau * (mass * q - at)
    # (where the largest value is so large that its neighbour is 64 and more below it, the kernels may take the others for nothing)
    dz_tol = 1.01 * tau * (mass * q * (q_rel + mass_rel) + at_tol + mass * 1e-18 + 1e-36) + 1e-37
    for train in (False, True):
        got_lse, got_loss, got_dz = distill(z, vocab, ids, t, tlse, tau, train)
        finite = lse.abs() < FLOAT_MAX
        assert_within(got_lse[finite], lse[finite], lse_tol[finite], ("lse", train))
        assert bool((got_lse[~finite] == -math.inf).all())
        shown = loss.abs() < FLOAT_MAX
        assert_within(got_loss[shown], loss[shown], loss_tol[shown], ("loss", train))
        assert bool((got_loss[~shown] == math.inf).all())
        if train:
            assert bool((got_dz[:, vocab:] == 0).all())
            assert_within(got_dz[:, :vocab], dz, dz_tol + (dz.abs() + dz_tol) * STEP[dtype], "dz")


def entries(z, vocab, k, seed):
    """Teacher entries: the student's first two columns of its largest value, and others anywhere."""
    g = gen(seed)
    ids = torch.stack([torch.randperm(vocab, device=DEV, generator=g)[:k] for _ in range(z.shape[0])])
    top = torch.sort(z[:, :vocab].float(), dim=1, descending=True, stable=True).indices[:, :2]
    ids = torch.where((ids[:, :, None] == top[:, None, :]).any(2), (top.max(1, keepdim=True).values + 1 + torch.arange(k, device=DEV)) % vocab, ids)
    ids[:, :2] = top
    t = 3.0 * torch.randn(ids.shape, device=DEV, generator=g) + 4.0
    t[:, 1] = t[:, 0] + 1e-6 * torch.arange(z.shape[0], device=DEV)
    return ids.to(torch.int32), t


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tau", TAUS)
@pytest.mark.parametrize("vocab", SIZES)
def test_distillation(dtype, tau, vocab):
    z = large_rows(vocab, dtype)
    ids, t = entries(z, vocab, 7, 2)
    check_distill(z, vocab, ids, t, tau)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tau", [1.0, 0.3, 50.0])
def test_distillation_against_the_teachers_own_sum(dtype, tau):
    vocab = 4096
    z = large_rows(vocab, dtype)
    ids, t = entries(z, vocab, 7, 3)
    check_distill(z, vocab, ids, t, tau, (torch.logsumexp(t.double() / as_float(tau), 1) + 0.25).float())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", SIZES)
def test_masked_columns_and_confident_rows(dtype, vocab):
    """Columns that the type's lowest value, -1e9 or -inf masks, and a row with one column far above: bounds of the columns that are left."""
    low = torch.finfo(TDT[dtype]).min
    z = torch.full((6, padded(vocab)), float("nan"), device=DEV, dtype=TDT[dtype])
    r = 3.0 * torch.randn((6, vocab), device=DEV, generator=gen(5))
    z[:, :vocab] = r.to(TDT[dtype])
    z[0, 9:vocab - 9] = low
    z[1, : vocab - 30] = -1e9
    z[2, 40:] = -math.inf
    z[2, vocab:] = math.nan
    z[3, vocab // 2] = 60.0
    z[4, :vocab] = low
    z[4, 17] = 5.0
    ids, t = entries(z, vocab, 5, 6)
    ids[2] = torch.arange(5, device=DEV)                # (what -inf masks would cost +inf)
    check_distill(z, vocab, ids, t, 1.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [2, 150, 600])
@pytest.mark.parametrize("mask", ["low", -1e9, -math.inf])
def test_log_sum_exp_beside_the_top_logits_of_masked_rows(dtype, rows, mask):
    """Most columns masked, the others anywhere in the row: the log-sum-exp is that of the others, to their bounds."""
    vocab, k = 40003, 6
    mask = torch.finfo(TDT[dtype]).min if mask == "low" else mask
    z = torch.full((rows, padded(vocab)), mask, device=DEV, dtype=TDT[dtype])
    left = torch.rand((rows, vocab), device=DEV, generator=gen(7)) < 0.01
    left[0], left[1] = False, False
    left[0, vocab - 9:], left[1, :9] = True, True
    z[:, :vocab] = torch.where(left, 3.0 * torch.randn((rows, vocab), device=DEV, generator=gen(8)), mask).to(TDT[dtype])
    ids, values, lse = torch.empty((rows, k), dtype=torch.int32, device=DEV), torch.empty((rows, k), device=DEV), torch.empty(rows, device=DEV)
    B.tide_topk_logits(rows, vocab, z, z.shape[1], k, 1.0, ids, values, lse, CODE[dtype], stream())
    sync()
    _, _, _, _, _, want, tol = statistics(z[:, :vocab], 1.0)
    assert float(want.abs().max()) < 60
    assert_within(lse, want, tol, "lse")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 5000, 33001, 128256, 200001])
def test_one_rule_for_infinities_and_nan(dtype, vocab):
    """The log-sum-exp of a row is NaN if the row holds a NaN, else +inf if it holds +inf, else -inf if it holds nothing else: in every operator, wherever
    in the row they stand."""
    inf, nan, at = math.inf, math.nan, [0, 9, vocab // 2, vocab - 1]
    z = torch.full((24, padded(vocab, 8)), nan, device=DEV, dtype=TDT[dtype])
    z[:, :vocab] = torch.randn((24, vocab), device=DEV, generator=gen(9)).to(TDT[dtype])
    row = 0
    for i in at:
        for j in at:
            if i != j:
                z[row, i], z[row, j] = nan, inf
                row += 1
    for i in at:
        z[row, i], z[row + 1, i] = nan, inf
        row += 2
    z[20, :vocab] = -inf
    z[21, :vocab] = -inf
    z[21, vocab - 1] = nan
    z[22, : vocab - 1], z[22, vocab - 1] = -inf, inf
    z[23, :vocab] = inf
    z[23, vocab // 3] = nan
    want = torch.logsumexp(z[:, :vocab].double(), 1)
    assert torch.equal(want.isnan(), z[:, :vocab].isnan().any(1)) and int((want == inf).sum()) == 5 and int((want == -inf).sum()) == 1
    k = 5
    ids, values, lse = torch.empty((24, k), dtype=torch.int32, device=DEV), torch.empty((24, k), device=DEV), torch.empty(24, device=DEV)
    B.tide_topk_logits(24, vocab, z, z.shape[1], k, 1.0, ids, values, lse, CODE[dtype], stream())
    t = torch.zeros((24, k), device=DEV)
    others = torch.arange(k, device=DEV, dtype=torch.int32).repeat(24, 1)
    for got in (lse, distill(z, vocab, others, t, None, 1.0, False)[0], distill(z, vocab, others, t, None, 1.0, True)[0]):
        assert_within(got, want.float(), 0.0, "lse")
    for train in (False, True):                          # (none of these rows has a softmax)
        _, loss, dz = distill(z, vocab, others, t, None, 1.0, train)
        assert bool(loss.isnan().all())
        assert dz is None or bool(dz[:, :vocab].isnan().all()) and bool((dz[:, vocab:] == 0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("given", [False, True], ids=["among k", "teacher_lse"])
@pytest.mark.parametrize("rows,vocab,k,tau", [(1, 8, 1, 1.0), (3, 100, 100, 0.5), (4, 4095, 16, 1.0), (115, 4096, 16, 1.0), (5, 32001, 64, 1.5), (7, 128256, 32, 2.0),
                                              (2, 152064, 128, 1.0), (3, 175003, 8, 1.0)])
def test_ordinary_rows_by_bounds_of_their_own(dtype, given, rows, vocab, k, tau):
    z = logits(rows, vocab, padded(vocab, 8), dtype, seed=vocab + k)
    g = gen(vocab)
    ids = torch.stack([torch.randperm(vocab, device=DEV, generator=g)[:k] for _ in range(rows)]).to(torch.int32)
    t = 3.0 * torch.randn((rows, k), device=DEV, generator=g) + 4.0
    check_distill(z, vocab, ids, t, tau, (torch.logsumexp(t.double() / as_float(tau), 1) + 0.4).float() if given else None)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("order", sorted(_orders(64).keys() if torch.cuda.is_available() else ["none"]))
@pytest.mark.parametrize("rows", [2, 200, 600])
def test_log_sum_exp_of_every_order(dtype, order, rows):
    """The sum runs against a shift that rises as the row is read: the orders that raise it often, late or never."""
    vocab, k = 9000, 37
    row = _orders(vocab)[order]
    z = torch.full((rows, padded(vocab)), math.nan, device=DEV, dtype=TDT[dtype])
    z[0::2, :vocab] = row.to(TDT[dtype])
    z[1::2, :vocab] = row.flip(0).to(TDT[dtype])
    ids, values, lse = torch.empty((rows, k), dtype=torch.int32, device=DEV), torch.empty((rows, k), device=DEV), torch.empty(rows, device=DEV)
    B.tide_topk_logits(rows, vocab, z, z.shape[1], k, 1.0, ids, values, lse, CODE[dtype], stream())
    sync()
    _, _, _, _, _, want, tol = statistics(z[:, :vocab], 1.0)
    assert_within(lse, want, tol, "lse")
