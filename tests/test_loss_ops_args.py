"""Refusals of the losses' entry points, before anything touches a device: a code and a message, never a launch."""
import ctypes
import re

import pytest

from paper_2602_05145_amd import binding as B

F32, BF16 = B.TIDE_DTYPE_FP32, B.TIDE_DTYPE_BF16
P = 4096          # an address that no call may look at


def topk(rows=4, vocab=100, z=P, ldz=104, k=8, temperature=1.0, ids=P, values=P, lse=P, dtype=BF16):
    return B.tide_topk_logits(rows, vocab, z, ldz, k, temperature, ids, values, lse, dtype, None, check=False)


def distill(train, rows=4, vocab=100, z=P, dz=P, ldz=104, k=8, ids=P, t=P, tlse=None, temperature=1.0, mask=P, lse=P, loss=P, dtype=BF16):
    if train:
        return B.tide_distill_train(rows, vocab, z, dz, ldz, k, ids, t, tlse, temperature, mask, lse, loss, dtype, None, check=False)
    return B.tide_distill_eval(rows, vocab, z, ldz, k, ids, t, tlse, temperature, mask, lse, loss, dtype, None, check=False)


def lm_fwd(rows=4, vocab=100, d=64, y=P, w=P, tokens=P, mask=P, lse=P, loss=P, dtype=BF16, ws=P, n=1 << 40):
    return B.tide_lm_ce_fwd(rows, vocab, d, y, w, tokens, mask, lse, loss, dtype, ws, n, None, check=False)


def lm_bwd(rows=4, vocab=100, d=64, y=P, w=P, tokens=P, mask=P, lse=P, weights=None, scale=1.0, dy=P, dw=P, dw_dtype=BF16, dtype=BF16, ws=P, n=1 << 40):
    return B.tide_lm_ce_bwd(rows, vocab, d, y, w, tokens, mask, lse, weights, scale, dy, dw, dw_dtype, dtype, ws, n, None, check=False)


BAD_LOGITS = [dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=-3), dict(ldz=96), dict(ldz=108), dict(ldz=(1 << 28) + 8), dict(z=P + 8), dict(dtype=2), dict(dtype=-1),
              dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=1e-7), dict(temperature=2e6), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(k=0), dict(k=-1), dict(k=129)]


@pytest.mark.parametrize("bad", BAD_LOGITS + [dict(vocab=7, k=8)], ids=str)
def test_topk_refuses(bad):
    assert topk(**bad) == B.TIDE_ERR_CONFIG and B.tide_last_error()


@pytest.mark.parametrize("bad", BAD_LOGITS + [dict(dz=P + 4)], ids=str)
def test_distill_refuses(bad):
    assert distill(True, **bad) == B.TIDE_ERR_CONFIG
    if "dz" not in bad:
        assert distill(False, **bad) == B.TIDE_ERR_CONFIG


def test_null_pointers_are_refused():
    for name in ("z", "ids", "values"):
        assert topk(**{name: None}) == B.TIDE_ERR_NULL, name
    for name in ("z", "dz", "ids", "t", "mask", "lse", "loss"):
        assert distill(True, **{name: None}) == B.TIDE_ERR_NULL, name
        if name != "dz":
            assert distill(False, **{name: None}) == B.TIDE_ERR_NULL, name
    for name in ("y", "w", "tokens", "mask", "lse", "loss", "ws"):
        assert lm_fwd(**{name: None}) == B.TIDE_ERR_NULL, name
    for name in ("y", "w", "tokens", "mask", "lse", "dy", "ws"):
        assert lm_bwd(**{name: None}) == B.TIDE_ERR_NULL, name
    assert topk(rows=0, z=None, ids=None, values=None, lse=None) == B.TIDE_OK          # nothing to do
    assert distill(True, rows=0, z=None, dz=None, ids=None, t=None, mask=None, lse=None, loss=None) == B.TIDE_OK
    assert distill(False, rows=0, z=None, ids=None, t=None, mask=None, lse=None, loss=None) == B.TIDE_OK
    assert topk(rows=0, z=None, k=0) == B.TIDE_ERR_CONFIG
    with pytest.raises(B.TideError):
        B.tide_topk_logits(1, 8, None, 8, 1, 1.0, P, P, None, F32, None)


BAD_HEADS = [dict(rows=0), dict(rows=-1), dict(rows=(1 << 22) + 1), dict(vocab=0), dict(vocab=1 << 21), dict(d=0), dict(d=1 << 21), dict(d=60), dict(vocab=7),
             dict(dtype=2), dict(y=P + 8), dict(w=P + 4)]


@pytest.mark.parametrize("bad", BAD_HEADS, ids=str)
def test_lm_ce_refuses(bad):
    assert lm_fwd(**bad) == B.TIDE_ERR_CONFIG
    assert lm_bwd(**bad) == B.TIDE_ERR_CONFIG
    if not {"y", "w"} & set(bad):
        s = dict(rows=4, vocab=100, d=64, dtype=BF16) | bad
        assert B.tide_lm_ce_workspace_bytes(s["rows"], s["vocab"], s["d"], s["dtype"]) == 0


def test_lm_ce_refuses_bad_outputs_and_workspaces():
    for bad in (dict(dy=P + 8), dict(dw=P + 8), dict(scale=float("nan")), dict(scale=float("inf")), dict(dw_dtype=3), dict(dtype=F32, dw_dtype=BF16)):
        assert lm_bwd(**bad) == B.TIDE_ERR_CONFIG, bad
    need = B.tide_lm_ce_workspace_bytes(4, 100, 64, BF16)
    assert need > 0
    for call in (lm_fwd, lm_bwd):
        assert call(n=need - 1) == B.TIDE_ERR_WORKSPACE and str(need) in B.tide_last_error()
        assert call(ws=P + 128) == B.TIDE_ERR_WORKSPACE


def test_more_rows_than_a_launch_holds_are_refused():
    for rows in (1 << 22, 1 << 23, 1 << 25):
        assert topk(rows=rows) == distill(True, rows=rows) == distill(False, rows=rows) == B.TIDE_ERR_CONFIG
    for rows, vocab in (((1 << 21) + 1, 8), (1 << 22, 8), (1 << 21, (1 << 16) + 8), (1 << 21, 128256), ((1 << 37) // 128256 + 1, 128256)):
        assert lm_fwd(rows=rows, vocab=vocab) == lm_bwd(rows=rows, vocab=vocab) == B.TIDE_ERR_CONFIG
        assert B.tide_lm_ce_workspace_bytes(rows, vocab, 64, BF16) == 0
    assert B.tide_lm_ce_workspace_bytes(1 << 20, 128256, 64, BF16) > 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [8, 1000, 32001, 128256])
def test_lm_ce_workspace_never_falls_as_rows_grow(dtype, vocab):
    """A workspace made for a number of rows serves every smaller one; and it does not grow with rows x vocab."""
    sizes = [B.tide_lm_ce_workspace_bytes(r, vocab, 264, dtype) for r in list(range(1, 5000, 7)) + list(range(5000, 70000, 997))]
    assert all(b >= a > 0 for a, b in zip(sizes, sizes[1:]))
    whole = B.tide_lm_ce_workspace_bytes(65536, vocab, 264, dtype)
    per_row = 264 * 16 + 8 * ((vocab + 255) // 256) + 256 * 4 + 64   # y, dy, its fp32 sums; statistics of 256 columns; narrowest piece
    assert whole <= (1 << 30) + (256 << 20) + 65536 * per_row


def test_header_documents_every_argument_of_the_bindings():
    """The ctypes signatures take as many arguments as the header's declarations."""
    text = open(re.sub(r"paper_2602_05145_amd.*", "include/tide_draft.h", B.LIB_PATH)).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for name in ("tide_topk_logits", "tide_distill_eval", "tide_distill_train", "tide_lm_ce_workspace_bytes", "tide_lm_ce_fwd", "tide_lm_ce_bwd"):
        args = re.search(name + r"\s*\(([^)]*)\)", text).group(1).split(",")
        f = getattr(B.lib(), name)
        assert len(args) == len(f.argtypes), name
        for a, t in zip(args, f.argtypes):
            assert ("*" in a) == (t is ctypes.c_void_p), (name, a)
            assert ("float" in a and "*" not in a) == (t is ctypes.c_float), (name, a)
