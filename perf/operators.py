"""The losses of a draft and what they are made from, as cases that can be timed one by one and held to their definitions.

Three operators: the largest logits of a row with its log-sum-exp (what a served target leaves to train on), distillation
from such logits (loss alone, or with the gradient of the student's logits), and cross-entropy of an LM head from the
hidden states, without keeping logits (loss alone, or with the gradients of hidden states and weight).  With `own` they are
the library's calls, through the names of `paper_2602_05145_amd.binding`; without it they are written out in torch, in 32 bits.
Widths and vocabularies come from the configurations of `paper_2602_05145_amd.workloads`, or are odd ones of that range.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}


def listed():
    return [
        # a target serving one request: the largest logits of its one new position (launches and latency count)
        dict(name="topk_one", kind="topk", dtype="bf16", rows=1, vocab=32000, k=8, temperature=1.0),
        # one verification round of a served batch: 15 requests with four positions each, and one without a draft
        dict(name="topk_verify", kind="topk", dtype="bf16", rows=61, vocab=128256, k=32, temperature=1.0),
        # fp32 logits of a prompt of odd length over an odd vocabulary, softened
        dict(name="topk_prompt_fp32", kind="topk", dtype="fp32", rows=1999, vocab=32001, k=64, temperature=2.0),
        # a captured batch, block by block
        dict(name="topk_8b", kind="topk", dtype="bf16", rows=8192, vocab=128256, k=32, temperature=1.0),
        # the fp32 configuration used to check a setup
        dict(name="distill_tiny_fp32", kind="distill", dtype="fp32", rows=128, vocab=4096, k=16, temperature=1.0, lse=False, grad=True, kept=115),
        # deployment gate: the loss alone on held-out requests, with the teacher's own log-sum-exp
        dict(name="distill_eval_8b", kind="distill", dtype="bf16", rows=3999, vocab=128256, k=20, temperature=1.0, lse=True, grad=False, kept=3400),
        # fp32 training rows over an odd vocabulary, many teacher logits
        dict(name="distill_fp32", kind="distill", dtype="fp32", rows=1665, vocab=32001, k=64, temperature=1.5, lse=False, grad=True, kept=1415),
        # one block of logits of the large draft, softened
        dict(name="distill_8b", kind="distill", dtype="bf16", rows=8192, vocab=128256, k=32, temperature=2.0, lse=False, grad=True, kept=6963),
        # the fp32 configuration used to check a setup: forward and backward
        dict(name="lm_ce_tiny_fp32", kind="lm_ce", dtype="fp32", rows=128, vocab=4096, d=256, grad=True, kept=115),
        # held-out loss of the large draft
        dict(name="lm_ce_eval_8b", kind="lm_ce", dtype="bf16", rows=3999, vocab=128256, d=4096, grad=False, kept=3400),
        # a few requests' adaptation step of the small draft
        dict(name="lm_ce_small", kind="lm_ce", dtype="bf16", rows=1665, vocab=32000, d=2048, grad=True, kept=1415),
        # a full batch of the large draft, 15 % of its positions prompt: forward and backward, the largest call
        dict(name="lm_ce_8b", kind="lm_ce", dtype="bf16", rows=32768, vocab=128256, d=4096, grad=True, kept=27853),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("topk", "distill", "lm_ce"))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    vocab = rng.choice((4096, 32000, 128256, 152064, _log_int(rng, 1000, 152064), _log_int(rng, 1000, 152064)))
    if kind == "lm_ce":
        d = 8 * _log_int(rng, 32, 640)
        rows = _log_int(rng, 1, 16384)
        most = 2e12 if dtype == "bf16" else 1e11
        rows = max(1, min(rows, int(most / (2.0 * vocab * d))))
        return dict(kind=kind, dtype=dtype, rows=rows, vocab=vocab, d=d, grad=rng.random() < 0.7, kept=max(1, int(rows * rng.uniform(0.6, 1.0))))
    rows = max(1, min(_log_int(rng, 1, 8192), (1 << 30) // vocab // (1 if dtype == "bf16" else 2)))
    k = _log_int(rng, 1, 128)
    temperature = rng.choice((1.0, 1.0, 0.7, 2.0, 4.0))
    if kind == "topk":
        return dict(kind=kind, dtype=dtype, rows=rows, vocab=vocab, k=k, temperature=temperature)
    return dict(kind=kind, dtype=dtype, rows=rows, vocab=vocab, k=k, temperature=temperature, lse=rng.random() < 0.4,
                grad=rng.random() < 0.7, kept=max(1, int(rows * rng.uniform(0.6, 1.0))))


def _stride(vocab):
    """Elements between two rows of logits: a multiple of 64, as the library's own blocks of logits have them."""
    return (vocab + 63) // 64 * 64


def _mask(case, g):
    """One byte per row, 1 where the row carries loss: case["kept"] of them."""
    mask = torch.zeros(case["rows"], dtype=torch.uint8, device=DEV)
    mask[torch.randperm(case["rows"], device=DEV, generator=g)[:case["kept"]]] = 1
    return mask


def _tokens(case, g):
    """Emitted tokens: frequent ids far more often than rare ones."""
    u = torch.rand(case["rows"], device=DEV, generator=g)
    return (case["vocab"] ** u - 1).to(torch.int32).clamp_(0, case["vocab"] - 1)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt, rows, vocab = DTYPE[case["dtype"]], case["rows"], case["vocab"]
    state = dict(case=case)
    if case["kind"] == "lm_ce":
        d = case["d"]
        # hidden states behind a norm, weights of a model's usual spread: logits of a few units
        state["y"] = (2.0 * torch.randn((rows, d), device=DEV, generator=g)).to(dt)
        state["w"] = (0.02 * torch.randn((vocab, d), device=DEV, generator=g)).to(dt)
        state["tokens"], state["mask"] = _tokens(case, g), _mask(case, g)
        state["lse"], state["loss_rows"] = (torch.empty(rows, device=DEV) for _ in range(2))
        if case["grad"]:
            state["dy"], state["dw"] = torch.empty_like(state["y"]), torch.empty_like(state["w"])
        return state
    k, ldz = case["k"], _stride(vocab)
    z = torch.empty((rows, ldz), device=DEV, dtype=dt)
    z[:, :vocab] = 2.0 * torch.randn((rows, vocab), device=DEV, generator=g)
    z[:, vocab:] = 0
    # a few columns far above the others, as a model that knows something has them
    first = torch.randint(0, vocab, (rows, 1), device=DEV, generator=g)
    step = torch.randint(1, max(2, vocab // k), (rows, 1), device=DEV, generator=g)
    ids = (first + step * torch.arange(k, device=DEV)) % vocab
    drops = -torch.log(torch.rand((rows, k), device=DEV, generator=g).clamp_(min=1e-6))
    peaks = 9.0 - 0.5 * drops.cumsum(1)
    z.scatter_add_(1, ids, peaks.clamp(min=0).to(dt))
    state["z"] = z
    if case["kind"] == "topk":
        state["ids"] = torch.empty((rows, k), dtype=torch.int32, device=DEV)
        state["values"], state["lse"] = torch.empty((rows, k), device=DEV), torch.empty(rows, device=DEV)
        return state
    state["teacher_ids"] = ids.to(torch.int32)
    state["teacher_logits"] = (peaks + 0.7 * torch.randn((rows, k), device=DEV, generator=g)).to(torch.bfloat16).float()
    state["teacher_lse"] = None
    if case["lse"]:   # of the teacher's whole row: some of its mass lies outside the k
        state["teacher_lse"] = torch.logsumexp(state["teacher_logits"] / case["temperature"], 1) + 0.3 * torch.rand(rows, device=DEV, generator=g)
    state["mask"] = _mask(case, g)
    state["lse"], state["loss_rows"] = (torch.empty(rows, device=DEV) for _ in range(2))
    if case["grad"]:
        state["dz"] = torch.empty_like(z)
    return state


def _code(case):
    from paper_2602_05145_amd import binding as B
    return B.TIDE_DTYPE_BF16 if case["dtype"] == "bf16" else B.TIDE_DTYPE_FP32


def _run_own(s):
    from paper_2602_05145_amd import binding as B
    case = s["case"]
    rows, vocab, code = case["rows"], case["vocab"], _code(case)
    stream = torch.cuda.current_stream().cuda_stream
    if case["kind"] == "topk":
        B.tide_topk_logits(rows, vocab, s["z"], s["z"].shape[1], case["k"], case["temperature"], s["ids"], s["values"], s["lse"], code, stream)
        return dict(ids=s["ids"], values=s["values"], lse=s["lse"])
    if case["kind"] == "distill":
        teacher = (case["k"], s["teacher_ids"], s["teacher_logits"], s["teacher_lse"], case["temperature"])
        if case["grad"]:
            B.tide_distill_train(rows, vocab, s["z"], s["dz"], s["z"].shape[1], *teacher, s["mask"], s["lse"], s["loss_rows"], code, stream)
            return dict(lse=s["lse"], loss_rows=s["loss_rows"], dz=s["dz"])
        B.tide_distill_eval(rows, vocab, s["z"], s["z"].shape[1], *teacher, s["mask"], s["lse"], s["loss_rows"], code, stream)
        return dict(lse=s["lse"], loss_rows=s["loss_rows"])
    if "workspace" not in s:   # a program keeps it for its next step
        s["workspace"] = torch.empty(B.tide_lm_ce_workspace_bytes(rows, vocab, case["d"], code), dtype=torch.uint8, device=DEV)
    ws = s["workspace"]
    B.tide_lm_ce_fwd(rows, vocab, case["d"], s["y"], s["w"], s["tokens"], s["mask"], s["lse"], s["loss_rows"], code, ws, ws.numel(), stream)
    if not case["grad"]:
        return dict(lse=s["lse"], loss_rows=s["loss_rows"])
    B.tide_lm_ce_bwd(rows, vocab, case["d"], s["y"], s["w"], s["tokens"], s["mask"], s["lse"], None, 1.0 / case["kept"], s["dy"], s["dw"], code,
                     code, ws, ws.numel(), stream)
    return dict(lse=s["lse"], loss_rows=s["loss_rows"], dy=s["dy"], dw=s["dw"])


def _plain_topk(s):
    case = s["case"]
    z = s["z"][:, :case["vocab"]].float() + 0.0          # (one zero, not two)
    bits = z.view(torch.int32).to(torch.int64)
    order = torch.where(bits < 0, -1 - (bits & 0x7FFFFFFF), bits)   # ascends as the values do
    key = order * 2 ** 32 + (case["vocab"] - 1 - torch.arange(case["vocab"], device=DEV))   # equal values: the lowest index first
    ids = torch.topk(key, case["k"], dim=1).indices
    a = z / case["temperature"]
    top = a.amax(1, keepdim=True)
    return dict(ids=ids.to(torch.int32), values=z.gather(1, ids), lse=top[:, 0] + torch.log(torch.exp(a - top).sum(1)))


def _plain_distill(s):
    case = s["case"]
    tau, ids = case["temperature"], s["teacher_ids"].long()
    a = s["z"][:, :case["vocab"]].float() / tau
    top = a.amax(1, keepdim=True)
    e = torch.exp(a - top)
    total = e.sum(1, keepdim=True)
    log_q = a.gather(1, ids) - top - torch.log(total)
    t = s["teacher_logits"] / tau
    if s["teacher_lse"] is None:
        t_top = t.amax(1, keepdim=True)
        log_p = t - t_top - torch.log(torch.exp(t - t_top).sum(1, keepdim=True))
    else:
        log_p = t - s["teacher_lse"][:, None]
    p = torch.exp(log_p)
    keep = s["mask"] != 0
    out = dict(lse=top[:, 0] + torch.log(total[:, 0]), loss_rows=torch.where(keep, tau * tau * (p * (log_p - log_q)).sum(1), 0.0))
    if case["grad"]:
        dz = torch.zeros(s["dz"].shape, device=DEV)
        dz[:, :case["vocab"]] = p.sum(1, keepdim=True) * (e / total)
        dz.scatter_add_(1, ids, -p)
        out["dz"] = (tau * dz * keep[:, None]).to(s["dz"].dtype)
    return out


def _plain_lm_ce(s):
    case = s["case"]
    rows, y, w = torch.arange(case["rows"], device=DEV), s["y"].float(), s["w"].float()
    tokens, keep = s["tokens"].long(), s["mask"] != 0
    z = y @ w.T
    top = z.amax(1, keepdim=True)
    label = z[rows, tokens] - top[:, 0]
    e = z.sub_(top).exp_()
    total = e.sum(1)
    lse = top[:, 0] + torch.log(total)
    out = dict(lse=torch.where(keep, lse, 0.0), loss_rows=torch.where(keep, torch.log(total) - label, 0.0))
    if case["grad"]:
        e /= total[:, None]
        e[rows, tokens] -= 1.0
        e *= (keep / case["kept"])[:, None]
        out["dy"], out["dw"] = (e @ w).to(s["dy"].dtype), (e.T @ y).to(s["dw"].dtype)
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"topk": _plain_topk, "distill": _plain_distill, "lm_ce": _plain_lm_ce}[state["case"]["kind"]](state)


def work(case):
    rows, vocab, es = case["rows"], case["vocab"], SIZE[case["dtype"]]
    if case["kind"] == "lm_ce":
        # a row without loss has nothing to compute; logits, and with gradients the two products behind them
        products = 2.0 * case["kept"] * vocab * case["d"]
        read = es * (case["kept"] + vocab) * case["d"] + 13.0 * rows
        return dict(bytes=read + (es * (rows + vocab) * case["d"] if case["grad"] else 0), flops=products * (3 if case["grad"] else 1))
    if case["kind"] == "topk":
        return dict(bytes=float(rows) * (vocab * es + 8 * case["k"] + 4), flops=4.0 * rows * vocab)
    kept = case["kept"] if case["grad"] else rows
    moved = float(rows) * vocab * es + (float(rows) * _stride(vocab) * es if case["grad"] else 0)
    return dict(bytes=moved + rows * (8.0 * case["k"] + 9), flops=4.0 * rows * vocab + (3.0 * kept * vocab if case["grad"] else 0))


def exact(case, seed):
    """The same outputs in 64 bits, row block by row block."""
    s = prepare(case, seed)
    rows, vocab = case["rows"], case["vocab"]
    blocks = [slice(r, min(rows, r + 1024)) for r in range(0, rows, 1024)]
    parts = []
    if case["kind"] == "topk":
        for b in blocks:
            z = s["z"][b, :vocab].double()
            values, ids = torch.sort(z, dim=1, descending=True, stable=True)
            parts.append(dict(ids=ids[:, :case["k"]].to(torch.int32), values=values[:, :case["k"]], lse=torch.logsumexp(z / case["temperature"], 1)))
    elif case["kind"] == "distill":
        for b in blocks:
            tau = float(case["temperature"])
            log_q = torch.log_softmax(s["z"][b, :vocab].double() / tau, 1)
            t, ids, keep = s["teacher_logits"][b].double() / tau, s["teacher_ids"][b].long(), s["mask"][b].double()
            norm = torch.logsumexp(t, 1) if s["teacher_lse"] is None else s["teacher_lse"][b].double()
            p = torch.exp(t - norm[:, None])
            part = dict(lse=torch.logsumexp(s["z"][b, :vocab].double() / tau, 1),
                        loss_rows=keep * tau ** 2 * (p * (t - norm[:, None] - log_q.gather(1, ids))).sum(1))
            if case["grad"]:
                dz = torch.exp(log_q) * p.sum(1, keepdim=True)
                dz = dz.scatter_add(1, ids, -p) * (tau * keep[:, None])
                part["dz"] = torch.nn.functional.pad(dz, (0, s["z"].shape[1] - vocab))
            parts.append(part)
    else:
        w, dw = s["w"].double(), None
        for b in blocks:
            y, tokens, keep = s["y"][b].double(), s["tokens"][b].long()[:, None], s["mask"][b].double()
            z = y @ w.T
            lse = torch.logsumexp(z, 1)
            part = dict(lse=keep * lse, loss_rows=keep * (lse - z.gather(1, tokens)[:, 0]))
            if case["grad"]:
                dz = torch.exp(z - lse[:, None])
                dz.scatter_add_(1, tokens, -torch.ones_like(dz[:, :1]))
                dz *= keep[:, None] / case["kept"]
                part["dy"] = dz @ w
                dw = dz.T @ y if dw is None else dw.addmm_(dz.T, y)
            parts.append(part)
        out = {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
        return dict(out, dw=dw) if case["grad"] else out
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
