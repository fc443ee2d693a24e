"""Refusals of embedding, AdamW and verification, before anything touches a device: a code and a message, never a launch."""
import ctypes
import re

import pytest
import torch

from paper_2602_05145_amd import binding as B

F32, BF16 = B.TIDE_DTYPE_FP32, B.TIDE_DTYPE_BF16
P = 4096          # an address that no call may look at
NAN, INF = float("nan"), float("inf")


def embed_fwd(rows=4, vocab=100, d=64, ids=P, table=P, scale=1.0, out=P, dtype=BF16):
    return B.tide_embed_fwd(rows, vocab, d, ids, table, scale, out, dtype, None, check=False)


def embed_bwd(rows=4, vocab=100, d=64, ids=P, dy=P, scale=1.0, dtable=P, dtable_dtype=F32, accumulate=0, dtype=BF16, ws=P, n=1 << 40):
    return B.tide_embed_bwd(rows, vocab, d, ids, dy, scale, dtable, dtable_dtype, accumulate, dtype, ws, n, None, check=False)


def verify(rows=5, requests=2, vocab=100, cu=P, target=P, ldt=104, draft=P, ldd=104, tokens=P, temperature=P, uniforms=P, accepted=P, out=P, dtype=BF16, ws=P, n=1 << 40):
    return B.tide_verify_drafts(rows, requests, vocab, cu, target, ldt, draft, ldd, tokens, temperature, uniforms, accepted, out, dtype, ws, n, None, check=False)


def entry(**kw):
    c = (B.TideAdamwTensor * 1)()
    for k, v in (dict(param=P, master=P, grad=P, m=P, v=P, m_scale=P, v_scale=P, n=10, weight_decay=0.0, param_dtype=BF16, grad_dtype=F32, state_bits=8) | kw).items():
        setattr(c[0], k, v)
    return c


def adamw(tensors=None, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=0, grad_scale=None, dev=False, **kw):
    tensors = entry(**kw) if tensors is None else tensors
    if dev:
        return B.tide_adamw_dev(tensors, P, P, beta1, beta2, eps, grad_scale, 1, P, None, check=False)
    return B.tide_adamw(tensors, lr, beta1, beta2, eps, step, grad_scale, 1, None, check=False)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=(1 << 21) + 1), dict(vocab=0), dict(vocab=1 << 21), dict(d=0), dict(d=1 << 21), dict(rows=1 << 21, d=8193),
                                 dict(scale=NAN), dict(scale=INF), dict(dtype=2), dict(ids=P + 2)], ids=str)
def test_embedding_refuses(bad):
    assert embed_fwd(**bad) == B.TIDE_ERR_CONFIG and B.tide_last_error()
    assert embed_bwd(**bad) == B.TIDE_ERR_CONFIG
    if not {"scale", "dtype", "ids"} & set(bad):
        s = dict(rows=4, vocab=100, d=64) | bad
        assert B.tide_embed_bwd_workspace_bytes(s["rows"], s["vocab"], s["d"]) == 0


def test_embedding_refuses_pointers_types_and_workspaces():
    for name in ("ids", "table", "out"):
        assert embed_fwd(**{name: None}) == B.TIDE_ERR_NULL, name
    for name in ("ids", "dy", "dtable", "ws"):
        assert embed_bwd(**{name: None}) == B.TIDE_ERR_NULL, name
    assert embed_fwd(table=P + 1) == embed_fwd(out=P + 1) == embed_fwd(dtype=F32, table=P + 2) == B.TIDE_ERR_CONFIG
    assert embed_bwd(dy=P + 1) == embed_bwd(dtable=P + 2) == embed_bwd(dtable_dtype=3) == embed_bwd(dtype=F32, dtable_dtype=BF16) == B.TIDE_ERR_CONFIG
    need = B.tide_embed_bwd_workspace_bytes(4, 100, 64)
    assert need > 0 and embed_bwd(n=need - 1) == B.TIDE_ERR_WORKSPACE and str(need) in B.tide_last_error()
    assert embed_bwd(ws=P + 128) == B.TIDE_ERR_WORKSPACE
    assert embed_fwd(rows=0, ids=None, table=None, out=None) == B.TIDE_OK
    assert embed_bwd(rows=0, ids=None, dy=None, accumulate=1) == B.TIDE_OK      # nothing to add, nothing to clear
    with pytest.raises(B.TideError):
        B.tide_embed_fwd(1, 8, 8, None, P, 1.0, P, F32, None)


@pytest.mark.parametrize("d", [8, 257, 512, 513, 4096, 1 << 20])
def test_embedding_workspace_never_falls_as_rows_grow(d):
    most = min(1 << 21, (1 << 34) // d)
    rows = sorted(r for r in set(range(0, 4000, 3)) | {most} | {int(1.07 ** k) for k in range(216)} if r <= most)
    sizes = [B.tide_embed_bwd_workspace_bytes(r, 1000, d) for r in rows]
    assert all(b >= a > 0 for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("dev", [False, True])
@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=(1 << 33) + 1), dict(param_dtype=2), dict(grad_dtype=-1), dict(state_bits=16), dict(weight_decay=-0.1), dict(weight_decay=NAN),
                                 dict(weight_decay=INF), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=NAN), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF),
                                 dict(grad_scale=P + 2), dict(master=P + 2), dict(param=P + 1), dict(grad=P + 2), dict(grad_dtype=BF16, grad=P + 1), dict(m_scale=P + 1),
                                 dict(state_bits=32, m=P + 2), dict(param_dtype=F32, param=P + 2)], ids=str)
def test_adamw_refuses(bad, dev):
    assert adamw(dev=dev, **bad) == B.TIDE_ERR_CONFIG and B.tide_last_error()


def test_adamw_refuses_pointers_and_schedules():
    for name in ("param", "master", "grad", "m", "v", "m_scale", "v_scale"):
        assert adamw(**{name: None}) == B.TIDE_ERR_NULL, name
    assert adamw(step=-1) == adamw(step=2 ** 63 - 1) == adamw(lr=NAN) == adamw(lr=INF) == B.TIDE_ERR_CONFIG
    assert B.lib().tide_adamw(1, None, 0.1, 0.9, 0.99, 1e-8, 0, None, 1, None) == B.TIDE_ERR_NULL
    assert B.lib().tide_adamw(-1, entry(), 0.1, 0.9, 0.99, 1e-8, 0, None, 1, None) == B.TIDE_ERR_CONFIG
    for missing in range(3):
        args = [None if k == missing else P for k in range(3)]
        assert B.tide_adamw_dev(entry(), args[0], args[1], 0.9, 0.99, 1e-8, None, 1, args[2], None, check=False) == B.TIDE_ERR_NULL
    for args in ((P + 2, P, P), (P, P + 4, P), (P, P, P + 8)):
        assert B.tide_adamw_dev(entry(), args[0], args[1], 0.9, 0.99, 1e-8, None, 1, args[2], None, check=False) == B.TIDE_ERR_CONFIG
    # nothing to do: no tensors, and tensors without elements
    assert B.lib().tide_adamw(0, None, 0.1, 0.9, 0.99, 1e-8, 0, None, 1, None) == B.TIDE_OK
    assert adamw(n=0, param=None, grad=None, m=None, v=None, master=None, m_scale=None, v_scale=None) == B.TIDE_OK
    # one bad tensor behind a good one is found before anything is enqueued
    two = (B.TideAdamwTensor * 2)()
    two[0], two[1] = entry()[0], entry(m=None)[0]
    assert adamw(two) == B.TIDE_ERR_NULL and "tensor 1" in B.tide_last_error()


def test_adamw_lists_are_checked():
    f, h, c = torch.zeros(300), torch.zeros(300, dtype=torch.bfloat16), torch.zeros(300, dtype=torch.float8_e4m3fn)
    good = dict(param=h, master=f, grad=h, m=c, v=c, m_scale=torch.zeros(2), v_scale=torch.zeros(2), weight_decay=0.1)
    t = B.make_adamw_tensors([good, dict(param=f, grad=f, m=f, v=f)])
    assert len(t) == 2 and t[0].n == 300 and t[0].state_bits == 8 and t[1].state_bits == 32 and t[1].weight_decay == 0.0
    assert (t[0].param_dtype, t[0].grad_dtype, t[1].param_dtype) == (BF16, BF16, F32) and t[1].master is None
    for bad in (dict(master=None), dict(m=f), dict(v_scale=None), dict(m_scale=torch.zeros(1)), dict(grad=f[:-1]), dict(grad=f.double()), dict(param=h[::2]), dict(v=None)):
        with pytest.raises(ValueError):
            B.make_adamw_tensors([good | bad])


@pytest.mark.parametrize("bad", [dict(rows=1), dict(requests=-1), dict(rows=(1 << 20) + 1), dict(vocab=0), dict(vocab=(1 << 28) + 8, ldt=1 << 30, ldd=1 << 30),
                                 dict(rows=1 << 20, vocab=(1 << 15) + 8, ldt=1 << 16, ldd=1 << 16), dict(ldt=96), dict(ldt=108), dict(ldd=96), dict(ldd=100),
                                 dict(ldt=(1 << 28) + 8), dict(ldd=(1 << 28) + 8), dict(dtype=2), dict(target=P + 8), dict(draft=P + 2), dict(cu=P + 2), dict(tokens=P + 1),
                                 dict(temperature=P + 2), dict(uniforms=P + 2), dict(accepted=P + 1), dict(out=P + 3)], ids=str)
def test_verification_refuses(bad):
    assert verify(**bad) == B.TIDE_ERR_CONFIG and B.tide_last_error()


def test_verification_refuses_pointers_and_workspaces():
    for name in ("cu", "target", "tokens", "uniforms", "accepted", "out", "ws"):
        assert verify(**{name: None}) == B.TIDE_ERR_NULL, name
    need = B.tide_verify_workspace_bytes(5, 2, 100)
    assert need > 0 and verify(n=need - 1) == B.TIDE_ERR_WORKSPACE and str(need) in B.tide_last_error()
    assert verify(ws=P + 128) == B.TIDE_ERR_WORKSPACE
    assert verify(rows=0, requests=0, cu=None, target=None, draft=None, tokens=None, temperature=None, uniforms=None, accepted=None, out=None, ws=None, n=0) == B.TIDE_OK
    assert B.tide_verify_workspace_bytes(1, 2, 100) == B.tide_verify_workspace_bytes(5, 2, 0) == 0


def test_header_documents_every_argument_of_the_bindings():
    text = open(re.sub(r"paper_2602_05145_amd.*", "include/tide_draft.h", B.LIB_PATH)).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for name in ("tide_embed_fwd", "tide_embed_bwd_workspace_bytes", "tide_embed_bwd", "tide_adamw", "tide_adamw_dev", "tide_verify_workspace_bytes", "tide_verify_drafts"):
        args = re.search(name + r"\s*\(([^)]*)\)", text).group(1).split(",")
        f = getattr(B.lib(), name)
        assert len(args) == len(f.argtypes), name
        for a, t in zip(args, f.argtypes):
            assert ("*" in a) == (t in (ctypes.c_void_p, ctypes.POINTER(B.TideAdamwTensor))), (name, a)
            assert ("float" in a and "*" not in a) == (t is ctypes.c_float), (name, a)
    fields = re.search(r"typedef struct tide_adamw_tensor \{(.*?)\}", text, flags=re.S).group(1)
    assert re.findall(r"(\w+)\s*[,;]", fields) == [n for n, _ in B.TideAdamwTensor._fields_]
