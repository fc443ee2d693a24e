"""tide_lm_ce_fwd / tide_lm_ce_bwd against the definition in 64 bits: odd vocabularies, pieces, rows without loss, frozen heads."""
import pytest
import torch

from paper_2602_05145_amd import binding as B
from tests.gpu_util import stream, sync
from tests.internal_gemm import NT, args, gemm_lm_height
from tests.loss_util import CODE, DEV, HALF, STEP, TDT, assert_within, gen, sum_rel

pytestmark = pytest.mark.gpu


def head(rows, vocab, d, dtype, seed, scale=1.0):
    g = gen(seed)
    y = torch.randn((rows, d), device=DEV, generator=g).to(TDT[dtype])
    w = (scale * 2.0 / d ** 0.5 * torch.randn((vocab, d), device=DEV, generator=g)).to(TDT[dtype])
    tokens = torch.randint(0, vocab, (rows,), device=DEV, generator=g).to(torch.int32)
    mask = (torch.rand(rows, device=DEV, generator=g) < 0.8).to(torch.uint8)
    mask[0] = 1
    return y, w, tokens, mask


def workspace(rows, vocab, d, dtype, fill=None):
    ws = torch.empty(B.tide_lm_ce_workspace_bytes(rows, vocab, d, CODE[dtype]) + 256, dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF if fill is None else fill)          # NaN wherever a call reads what it has not written
    return ws


def call(y, w, tokens, mask, weights=None, scale=1.0, dw_dtype=None, want_dw=True, ws=None, guard=2):
    (rows, d), vocab = y.shape, w.shape[0]
    dtype = "bf16" if y.dtype == torch.bfloat16 else "fp32"
    ws = workspace(rows, vocab, d, dtype) if ws is None else ws
    need = B.tide_lm_ce_workspace_bytes(rows, vocab, d, CODE[dtype])
    behind = ws[need:].clone()
    lse, loss = (torch.full((rows + guard,), -7.0, device=DEV) for _ in range(2))
    B.tide_lm_ce_fwd(rows, vocab, d, y, w, tokens, mask, lse, loss, CODE[dtype], ws, need, stream())
    dw_dtype = dw_dtype or dtype
    dy = torch.full((rows + guard, d), -7.0, device=DEV, dtype=y.dtype)
    dw = torch.full((vocab + guard, d), -7.0, device=DEV, dtype=TDT[dw_dtype]) if want_dw else None
    B.tide_lm_ce_bwd(rows, vocab, d, y, w, tokens, mask, lse, weights, scale, dy, dw, CODE[dw_dtype], CODE[dtype], ws, need, stream())
    sync()
    for x, n in ((lse, rows), (loss, rows), (dy, rows), (dw, vocab)):
        assert x is None or bool((x[n:] == -7).all())
    assert torch.equal(ws[need:], behind)
    return lse[:rows], loss[:rows], dy[:rows], dw[:vocab] if want_dw else None


def reference(y, w, tokens, mask, weights, scale, dtype):
    """Each output with a bound: products of d terms, then a softmax, then (bf16) dz to bf16, then products of its rows or columns."""
    vocab, d = w.shape
    keep = (mask != 0) & (tokens >= 0) & (tokens < vocab)
    Y, W = torch.where(keep[:, None], y.double(), 0.0), w.double()
    z = Y @ W.T
    ez = (d + 2) * HALF * float((Y.abs() @ W.abs().T).max())          # a logit's error: d roundings of what its terms add up to
    lse = torch.logsumexp(z, 1)
    at = torch.where(keep, tokens, 0).long()[:, None]
    reach = float(z.abs().max())
    lse_tol = ez + sum_rel(vocab, reach) + 4 * HALF * (reach + 16)
    loss = lse - z.gather(1, at)[:, 0]
    g = torch.where(keep, (weights.double() if weights is not None else 1.0), 0.0)[:, None]
    dz = torch.exp(z - lse[:, None])
    dz_tol = dz * (2 * ez + lse_tol + sum_rel(vocab, reach) + 8 * HALF * (reach + 16)) + 2 * HALF
    dz.scatter_add_(1, at, -torch.ones_like(dz[:, :1]))
    dz, dz_tol = g * dz, g.abs() * dz_tol
    dz_tol = dz_tol + STEP[dtype] * (dz.abs() + dz_tol)
    a = abs(scale)
    dy = scale * (dz @ W)
    dy_tol = a * (dz_tol @ W.abs() + (vocab + 8) * HALF * (dz.abs() @ W.abs()))
    dw = scale * (dz.T @ Y)
    dw_tol = a * (dz_tol.T @ Y.abs() + (y.shape[0] + 8) * HALF * (dz.abs().T @ Y.abs()))
    zero = torch.zeros_like(lse)
    return ((torch.where(keep, lse, zero), lse_tol), (torch.where(keep, loss, zero), lse_tol + ez + 4 * HALF * (reach + 16)), (dy, dy_tol), (dw, dw_tol))


def check(y, w, tokens, mask, weights=None, scale=1.0, dw_dtype=None, want_dw=True):
    dtype = "bf16" if y.dtype == torch.bfloat16 else "fp32"
    got = call(y, w, tokens, mask, weights, scale, dw_dtype, want_dw)
    ref = reference(y, w, tokens, mask, weights, scale, dtype)
    stored = (0, 0, STEP[dtype], STEP[dw_dtype or dtype])
    for x, (want, tol), name, step in zip(got, ref, ("lse", "loss", "dy", "dw"), stored):
        if x is not None:
            tol = torch.as_tensor(tol, dtype=torch.float64, device=DEV)
            assert_within(x, want, tol + step * (want.abs() + tol) + 1e-37, name)
            if name in ("dy", "dw") and float(want.norm()) > 0:
                # the bounds above let every rounding be at its worst; taken together they are random
                off = float((x.double() - want).norm() / want.norm())
                assert off < (2.0 ** -8 if dtype == "bf16" else 1e-5), (name, off)
    return got


SHAPES = [(1, 8, 8), (1, 1000, 64), (2, 9, 8), (3, 255, 72), (5, 257, 64), (64, 264, 264), (129, 1003, 264), (300, 4096, 256), (257, 5003, 520), (1415, 2049, 128),
          (37, 32001, 192), (700, 9000, 1000)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,d", SHAPES)
def test_against_64_bits(dtype, rows, vocab, d):
    y, w, tokens, mask = head(rows, vocab, d, dtype, seed=rows + vocab + d)
    check(y, w, tokens, mask, scale=1.0 / max(1, int(mask.sum())))


@pytest.mark.parametrize("rows,vocab,d", [(1, 1, 1), (3, 2, 5), (4, 7, 3), (33, 101, 37), (130, 1001, 77)])
def test_fp32_takes_any_width(rows, vocab, d):
    check(*head(rows, vocab, d, "fp32", seed=d), scale=0.5)


@pytest.mark.parametrize("tail", range(8))
def test_vocabularies_of_every_remainder(tail):
    """bf16 products contract over eight columns at a time: the last ones reach back."""
    check(*head(70, 1000 + tail, 136, "bf16", seed=tail))


@pytest.mark.parametrize("dtype,rows,vocab,d", [("bf16", 30000, 40001, 64), ("bf16", 30000, 36000, 72), ("fp32", 20000, 20001, 20), ("bf16", 4099, 300007, 64)])
def test_several_pieces(dtype, rows, vocab, d):
    """Rows x vocabulary beyond what one piece holds; the reference by rows, dw summed over them."""
    y, w, tokens, mask = head(rows, vocab, d, dtype, seed=vocab)
    lse, loss, dy, dw = call(y, w, tokens, mask, scale=1.0 / rows)
    want_dw, worst = torch.zeros((vocab, d), dtype=torch.float64, device=DEV), 0.0
    for r in range(0, rows, 2000):
        b = slice(r, min(rows, r + 2000))
        ref = reference(y[b], w, tokens[b], mask[b], None, 1.0 / rows, dtype)
        assert_within(lse[b], *ref[0], "lse")
        assert_within(loss[b], *ref[1], "loss")
        assert_within(dy[b], ref[2][0], ref[2][1] + STEP[dtype] * (ref[2][0].abs() + ref[2][1]) + 1e-37, "dy")
        want_dw += ref[3][0]
    off = float((dw.double() - want_dw).norm() / want_dw.norm())
    assert off < (2.0 ** -8 if dtype == "bf16" else 1e-5), off
    by_row = (dw.double() - want_dw).norm(dim=1) / (want_dw.norm(dim=1) + 1e-4 * want_dw.norm())
    assert float(by_row.max()) < (2.0 ** -6 if dtype == "bf16" else 1e-4), int(by_row.argmax())   # no row of a piece's edge is wrong


HEIGHTS = [(100, 5003, 128, 128), (500, 3000, 64, 128), (1025, 9001, 64, 192), (700, 16000, 128, 192), (2100, 9001, 64, 256), (900, 16000, 128, 256), (200, 3001, 72, 128), (2100, 9001, 72, 256)]


@pytest.mark.parametrize("rows,vocab,d,height", HEIGHTS)
def test_every_height_of_tiles(rows, vocab, d, height):
    """Tiles of 128, 192 and 256 rows, 128 and 256 also over a width that is no whole number of slabs; every row kept, and a few."""
    assert gemm_lm_height(args(NT, rows, vocab, d)) == height
    y, w, tokens, mask = head(rows, vocab, d, "bf16", seed=rows)
    mask[:] = 1
    check(y, w, tokens, mask)
    mask[rows // 3:] = 0
    check(y, w, tokens, mask)


# both gradients in one pass up to four rows; not with five, a width that is no multiple of four, or a very wide head
@pytest.mark.parametrize("rows,vocab,d", [(1, 1, 4), (1, 1001, 256), (2, 63, 260), (3, 4099, 1028), (4, 257, 12), (4, 9001, 2052), (5, 1001, 256), (3, 300, 258), (2, 300, 16388), (17, 13001, 64), (32, 13001, 66)])
def test_fp32_few_rows(rows, vocab, d):
    check(*head(rows, vocab, d, "fp32", seed=rows + d), scale=0.5)


# the gradient of the hidden states as 32 sums over the vocabulary, of which the last are empty; 5; 2; and one of 4100 rows
@pytest.mark.parametrize("rows,vocab,d", [(1, 4097, 264), (115, 4096, 256), (70, 16389, 33), (65, 4099, 2056), (333, 700, 64), (130, 300, 72), (4100, 300, 1536)])
def test_fp32_sums_over_parts_of_the_vocabulary(rows, vocab, d):
    check(*head(rows, vocab, d, "fp32", seed=vocab), scale=0.25)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [7, 8, 9, 1024, 8191, 8192, 8193, 9216, 20481])
@pytest.mark.parametrize("pattern", ["all", "none", "last", "first", "every third", "not the first thousands"])
def test_kept_rows_are_found_in_any_number(dtype, rows, pattern):
    """Up to 8192 rows the blocks count what lies before them by themselves, beyond from counts of 1024 each."""
    y, w, tokens, mask = head(rows, 64, 8, dtype, seed=rows)
    i = torch.arange(rows, device=DEV)
    keep = {"all": i >= 0, "none": i < 0, "last": i == rows - 1, "first": i == 0, "every third": i % 3 == 1, "not the first thousands": i >= rows // 2}[pattern]
    mask.copy_(keep.to(torch.uint8))
    check(y, w, tokens, mask)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 5001])
def test_rows_without_loss_may_hold_anything(dtype, vocab):
    rows, d = 40, 64
    y, w, tokens, mask = head(rows, vocab, d, dtype, seed=3)
    mask[:] = 1
    mask[5], mask[6], mask[39] = 0, 0, 0
    tokens[7], tokens[8], tokens[9] = -1, vocab, 2 ** 31 - 1
    for r in (5, 6, 7, 8, 9, 39):
        y[r] = float("nan") if r % 2 else float("inf")
    lse, loss, dy, dw = check(y, w, tokens, mask)
    for r in (5, 6, 7, 8, 9, 39):
        assert lse[r] == 0 and loss[r] == 0 and bool((dy[r] == 0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 1003])
def test_no_row_has_loss(dtype, vocab):
    y, w, tokens, mask = head(20, vocab, 64, dtype, seed=4)
    mask[:] = 0
    for out in call(y, w, tokens, mask):
        assert bool((out == 0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_weights_scale_frozen_head_and_float_gradients(dtype):
    y, w, tokens, mask = head(90, 777, 128, dtype, seed=5)
    weights = torch.randn(90, device=DEV, generator=gen(6))
    weights[3] = 0.0
    a = check(y, w, tokens, mask, weights, scale=-0.25, dw_dtype="fp32")
    b = check(y, w, tokens, mask, weights, scale=-0.25, want_dw=False)
    assert all(torch.equal(p, q) for p, q in zip(a[:3], b[:3]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_confident_rows_and_large_logits(dtype):
    """Logits of hundreds, a label that takes all of the mass, one that takes none of it."""
    y, w, tokens, mask = head(50, 1200, 64, dtype, seed=7, scale=30.0)
    z = y.float() @ w.float().T
    tokens[:25] = z[:25].argmax(1).to(torch.int32)
    tokens[25:] = z[25:].argmin(1).to(torch.int32)
    lse, loss, dy, dw = check(y, w, tokens, mask)
    assert float(loss.max()) > 200 and bool(dy.isfinite().all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_same_bits_every_time_and_in_any_workspace(dtype):
    y, w, tokens, mask = head(333, 5003, 264, dtype, seed=8)
    a = call(y, w, tokens, mask)
    b = call(y, w, tokens, mask, ws=workspace(333, 5003, 264, dtype, fill=0))
    c = call(y, w, tokens, mask, ws=workspace(1000, 5003, 264, dtype, fill=0x7F))     # one that was made for more rows
    for x, p, q in zip(a, b, c):
        assert torch.equal(x, p) and torch.equal(x, q)


def test_gradients_against_differences():
    """Central differences of the mean loss in 64 bits."""
    rows, vocab, d, h = 5, 12, 8, 1e-4
    y, w, tokens, mask = head(rows, vocab, d, "fp32", seed=9)
    mask[2] = 0
    weights = torch.rand(rows, device=DEV, generator=gen(1)) + 0.5
    _, _, dy, dw = call(y, w, tokens, mask, weights, scale=0.2)

    def loss(Y, W):
        z = Y @ W.T
        return 0.2 * (mask * weights * (torch.logsumexp(z, 1) - z.gather(1, tokens.long()[:, None])[:, 0])).sum()

    Y, W = y.double(), w.double()
    for x, grad, f in ((Y, dy, lambda v: loss(v, W)), (W, dw, lambda v: loss(Y, v))):
        for i in range(x.shape[0]):
            for j in range(x.shape[1]):
                e = torch.zeros_like(x)
                e[i, j] = h
                assert abs(float((f(x + e) - f(x - e)) / (2 * h)) - float(grad[i, j])) < 1e-5
