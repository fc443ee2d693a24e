"""The losses as a program uses them: a target's top logits captured, a draft's head trained on them and on the emitted tokens, on a stream of
its own and replayed from a graph."""
import pytest
import torch

from paper_2602_05145_amd import binding as B
from tests.gpu_util import cosine, stream, sync, to_host
from tests.loss_util import CODE, DEV, TDT, gen

pytestmark = pytest.mark.gpu


class Program:
    """One adaptation step of a draft's LM head: hidden states and the target's logits in, losses and gradients out."""

    def __init__(self, dtype, rows=200, vocab=3000, d=256, k=16, tau=1.5, seed=1):
        g = gen(seed)
        self.dtype, self.rows, self.vocab, self.d, self.k, self.tau, self.code = dtype, rows, vocab, d, k, tau, CODE[dtype]
        dt = TDT[dtype]
        self.y = torch.randn((rows, d), device=DEV, generator=g).to(dt)
        self.w = (2 / d ** 0.5 * torch.randn((vocab, d), device=DEV, generator=g)).to(dt)
        self.target = (3 * torch.randn((rows, vocab), device=DEV, generator=g)).to(dt)
        self.mask = (torch.rand(rows, device=DEV, generator=g) < 0.85).to(torch.uint8)
        self.scale = 1.0 / max(1, int(self.mask.sum()))
        f = lambda *s: torch.zeros(s, device=DEV)
        self.ids, self.values, self.tlse = torch.zeros((rows, k), dtype=torch.int32, device=DEV), f(rows, k), f(rows)
        self.z = torch.zeros((rows, vocab), device=DEV, dtype=dt)
        self.lse, self.loss, self.ce_lse, self.ce_loss = f(rows), f(rows), f(rows), f(rows)
        self.dy, self.dw, self.ce_dy, self.ce_dw = (torch.zeros(s, device=DEV, dtype=dt) for s in ((rows, d), (vocab, d)) * 2)
        self.tokens = torch.zeros(rows, dtype=torch.int32, device=DEV)
        self.ws = torch.zeros(B.tide_lm_ce_workspace_bytes(rows, vocab, d, self.code), dtype=torch.uint8, device=DEV)

    def step(self):
        s = torch.cuda.current_stream().cuda_stream
        R, V, d, c = self.rows, self.vocab, self.d, self.code
        B.tide_topk_logits(R, V, self.target, V, self.k, self.tau, self.ids, self.values, self.tlse, c, s)
        self.tokens.copy_(self.ids[:, 0])
        B.tide_gemm(B.LAYOUT_NT, R, V, d, 1.0, self.y, self.w, self.z, None, c, c, 0, s)
        B.tide_distill_train(R, V, self.z, self.z, V, self.k, self.ids, self.values, self.tlse, self.tau, self.mask, self.lse, self.loss, c, s)
        B.tide_gemm(B.LAYOUT_NN, R, d, V, self.scale, self.z, self.w, self.dy, None, c, c, 0, s)
        B.tide_gemm(B.LAYOUT_TN, V, d, R, self.scale, self.z, self.y, self.dw, None, c, c, 0, s)
        B.tide_lm_ce_fwd(R, V, d, self.y, self.w, self.tokens, self.mask, self.ce_lse, self.ce_loss, c, self.ws, self.ws.numel(), s)
        B.tide_lm_ce_bwd(R, V, d, self.y, self.w, self.tokens, self.mask, self.ce_lse, None, self.scale, self.ce_dy, self.ce_dw, c, c, self.ws,
                         self.ws.numel(), s)

    def out(self):
        return [x.clone() for x in (self.ids, self.values, self.tlse, self.lse, self.loss, self.dy, self.dw, self.ce_lse, self.ce_loss, self.ce_dy, self.ce_dw)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_step_against_autograd_in_64_bits(dtype):
    p = Program(dtype)
    p.step()
    sync()
    y, w = p.y.double().requires_grad_(True), p.w.double().requires_grad_(True)
    z, keep, tau = y @ w.T, p.mask.double(), p.tau
    t = torch.log_softmax(p.target.double() / tau, 1)
    ids = t.topk(p.k, 1).indices
    log_p = t.gather(1, ids)
    kd = tau ** 2 * (log_p.exp() * (log_p - torch.log_softmax(z / tau, 1).gather(1, ids))).sum(1) * keep
    kd_dy, kd_dw = torch.autograd.grad(kd.sum() * p.scale, (y, w), retain_graph=True)
    ce = -torch.log_softmax(z, 1)[torch.arange(p.rows, device=DEV), p.target.double().argmax(1)] * keep
    ce_dy, ce_dw = torch.autograd.grad(ce.sum() * p.scale, (y, w))
    loose = 2e-2 if dtype == "bf16" else 1e-5         # (the distillation's logits are stored in the mode's type)
    for got, want in ((p.loss, kd), (p.ce_loss, ce)):
        assert float((got.double() - want.detach()).abs().max()) <= loose * (1 + float(want.detach().abs().max()))
    for got, want in ((p.dy, kd_dy), (p.dw, kd_dw), (p.ce_dy, ce_dy), (p.ce_dw, ce_dw)):
        assert cosine(to_host(got), want.detach().cpu().numpy()) > (0.9998 if dtype == "bf16" else 1 - 1e-9)
        assert float((got.double() - want.detach()).norm() / want.norm()) < (1e-2 if dtype == "bf16" else 1e-5)


@pytest.mark.parametrize("dtype,vocab", [("fp32", 3000), ("bf16", 3000), ("bf16", 40000), ("fp32", 40000), ("bf16", 128256), ("bf16", 140000)])
def test_captured_and_replayed(dtype, vocab):
    """Every replay, with new inputs and eager work between them, gives the eager call's bits; two captured programs do not meet."""
    progs = [Program(dtype, vocab=vocab, seed=s) for s in (1, 2)]
    eager = Program(dtype, vocab=vocab, seed=3)
    side = torch.cuda.Stream()
    graphs = []
    for p in progs:
        p.step()                                      # once before the capture
        sync()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            p.step()
        graphs.append(g)
    for turn in range(3):
        for i, p in enumerate(progs):
            q = Program(dtype, vocab=vocab, seed=10 * turn + i)
            p.y.copy_(q.y)
            p.target.copy_(q.target)
            p.mask.copy_(q.mask)
            p.w.copy_(q.w)
            q.scale = p.scale
            q.step()
            sync()
            for x in (p.dw, p.ce_dw, p.z, p.lse, p.ce_loss):
                x.fill_(float("nan"))
            graphs[i].replay()
            eager.step()
            graphs[i].replay()
            sync()
            for a, b in zip(p.out(), q.out()):
                assert torch.equal(a, b)


def test_on_a_stream_of_its_own_beside_other_work():
    a, b, c = (Program("bf16", seed=5) for _ in range(3))
    a.step()
    sync()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    s1.wait_stream(torch.cuda.current_stream())
    s2.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(s1):
            b.step()
        with torch.cuda.stream(s2):
            c.step()
    sync()
    for x, p, q in zip(a.out(), b.out(), c.out()):
        assert torch.equal(x, p) and torch.equal(x, q)
