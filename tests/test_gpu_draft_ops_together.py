"""A draft of the caller's own, built from the library's blocks: tokens embedded, normalised, scored by the same table (tied head), trained on the target's tokens by AdamW with 8-bit
moments, in one captured graph; and the round it is for, its drafts verified against a target and the acceptance handed to the controller."""
import pytest
import torch

from paper_2602_05145_amd import control as K
from tests.draft_ops_util import B, CODE, DEV, HALF, TDT, gen, room, run_verify, verify_ref

pytestmark = pytest.mark.gpu

ROWS, VOCAB, D, SCALE, EPS = 300, 504, 64, 8.0, 1e-5


class Draft:
    def __init__(self, dtype, seed):
        g = gen(seed)
        self.dtype, self.code, t = dtype, CODE[dtype], TDT[dtype]
        master = dict(table=0.1 * torch.randn((VOCAB, D), device=DEV, generator=g), gain=1 + 0.1 * torch.randn(D, device=DEV, generator=g))
        self.master = master if dtype == "bf16" else None
        self.param = {k: x.to(t) if dtype == "bf16" else x for k, x in master.items()}
        self.grad = {k: torch.zeros(x.shape, device=DEV) for k, x in master.items()}
        n = VOCAB * D
        self.m = dict(table=torch.zeros(n, dtype=torch.float8_e4m3fn, device=DEV), gain=torch.zeros(D, device=DEV))
        self.v = dict(table=torch.zeros(n, dtype=torch.float8_e4m3fn, device=DEV), gain=torch.zeros(D, device=DEV))
        self.scales = torch.zeros((2, (n + 255) // 256), device=DEV)
        self.lr, self.step, self.schedule = torch.tensor([1e-2], device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV), torch.empty(4, device=DEV)
        self.ids, self.labels = torch.zeros(ROWS, dtype=torch.int32, device=DEV), torch.zeros(ROWS, dtype=torch.int32, device=DEV)
        self.mask = torch.ones(ROWS, dtype=torch.uint8, device=DEV)
        self.x, self.y, self.dy, self.dx = (torch.empty((ROWS, D), dtype=t, device=DEV) for _ in range(4))
        self.rstd, self.lse, self.loss = (torch.empty(ROWS, device=DEV) for _ in range(3))
        self.lm_ws = room(B.tide_lm_ce_workspace_bytes(ROWS, VOCAB, D, self.code))
        self.embed_ws = room(B.tide_embed_bwd_workspace_bytes(ROWS, VOCAB, D))
        self.norm_ws = room(B.tide_rmsnorm_bwd_scratch_bytes(ROWS, D))
        row = lambda k, **kw: dict(param=self.param[k], master=self.master and self.master[k], grad=self.grad[k], m=self.m[k], v=self.v[k], **kw)   # noqa: E731
        self.listed = B.make_adamw_tensors([row("table", m_scale=self.scales[0], v_scale=self.scales[1], weight_decay=0.1), row("gain")])

    def forward(self, ids):
        s = torch.cuda.current_stream().cuda_stream
        B.tide_embed_fwd(ROWS, VOCAB, D, ids, self.param["table"], SCALE, self.x, self.code, s)
        B.tide_rmsnorm_fwd(ROWS, D, self.x, self.param["gain"], EPS, self.y, self.rstd, self.code, s)

    def train(self, update=True):
        s = torch.cuda.current_stream().cuda_stream
        self.forward(self.ids)
        w, g = self.param["table"], self.grad
        B.tide_lm_ce_fwd(ROWS, VOCAB, D, self.y, w, self.labels, self.mask, self.lse, self.loss, self.code, self.lm_ws, self.lm_ws.numel(), s)
        B.tide_lm_ce_bwd(ROWS, VOCAB, D, self.y, w, self.labels, self.mask, self.lse, None, 1.0 / ROWS, self.dy, g["table"], CODE["fp32"], self.code, self.lm_ws, self.lm_ws.numel(), s)
        B.tide_rmsnorm_bwd(ROWS, D, self.dy, self.x, self.param["gain"], self.rstd, None, self.dx, g["gain"], self.norm_ws, self.code, s)
        B.tide_embed_bwd(ROWS, VOCAB, D, self.ids, self.dx, SCALE, g["table"], CODE["fp32"], True, self.code, self.embed_ws, self.embed_ws.numel(), s)   # on top of the head's
        if update:
            B.tide_adamw_dev(self.listed, self.lr, self.step, 0.9, 0.99, 1e-8, None, 5, self.schedule, s)

    def logits(self, ids):
        self.forward(ids)
        ld = (VOCAB + 7) // 8 * 8
        z = torch.empty((ROWS, ld), dtype=TDT[self.dtype], device=DEV)
        B.tide_gemm(0, ROWS, VOCAB, D, 1.0, self.y, self.param["table"], z, None, self.code, self.code, False, torch.cuda.current_stream().cuda_stream)
        return z

    def state(self):
        got = dict(self.param) | {"grad_" + k: x for k, x in self.grad.items()} | {"m_" + k: x for k, x in self.m.items()} | {"v_" + k: x for k, x in self.v.items()}
        return got | dict(scales=self.scales, step=self.step, loss=self.loss)


def batch(draft, seed):
    g = gen(seed)
    ids = (VOCAB ** torch.rand(ROWS, device=DEV, generator=g) - 1).to(torch.int32)
    ids[-9:] = -1                                        # what pads a batch
    draft.ids.copy_(ids)
    draft.labels.copy_((ids.clamp(min=0) * 7 + 3) % VOCAB)
    draft.mask.fill_(1)
    draft.mask[-9:] = 0


def test_gradients_of_the_tied_table():
    """Of the sum of both uses, against 64-bit autograd: contractions over up to 504 terms, norms and a softmax in fp32, 2 (504 + 300 + 64) half steps for the whole in the 2-norm."""
    d = Draft("fp32", 1)
    batch(d, 2)
    d.train(update=False)
    table, gain = (d.param[k].double().requires_grad_() for k in ("table", "gain"))
    fine = d.ids >= 0
    x = SCALE * table[d.ids[fine].long()]
    y = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * gain
    loss = torch.nn.functional.cross_entropy(y @ table.T, d.labels[fine].long(), reduction="sum") / ROWS
    loss.backward()
    tol = 2 * (VOCAB + ROWS + D) * HALF
    assert abs(float(d.loss.double().sum()) / ROWS - float(loss)) <= tol * float(loss)
    for got, want in ((d.grad["table"], table.grad), (d.grad["gain"], gain.grad)):
        assert float((got.double() - want).norm()) <= tol * float(want.norm())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_training_step_captured_and_replayed(dtype):
    """Four replays with new tokens, eager steps of another draft between them; each leaves what the eager step leaves, bit for bit."""
    a, b, other = Draft(dtype, 3), Draft(dtype, 3), Draft(dtype, 4)
    batch(other, 5)
    other.train()                                        # (the first calls on a device set function attributes)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.train()
    for k in range(4):
        batch(a, 10 + k), batch(b, 10 + k)
        a.train()
        graph.replay()
        other.train()
        torch.cuda.synchronize()
        for (name, x), y in zip(a.state().items(), b.state().values()):
            assert torch.equal(x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x, y.view(torch.uint8) if y.dtype == torch.float8_e4m3fn else y), (k, name)
    assert int(b.step) == 4


def test_a_round_of_drafts_reaches_the_controller():
    """Target and draft logits made by the library, tokens drawn from the draft's, verified; the acceptance of each request is what the controller observes."""
    target, draft = Draft("bf16", 7), Draft("bf16", 8)
    requests, n = 60, 4
    g = gen(9)
    ids = torch.randint(0, VOCAB, (ROWS,), device=DEV, generator=g, dtype=torch.int32)
    z_t, z_d = target.logits(ids), draft.logits(ids)
    cu = torch.arange(0, ROWS + 1, n + 1, dtype=torch.int32, device=DEV)
    drafted = (torch.arange(ROWS, device=DEV) % (n + 1) != n).nonzero()[:, 0]
    z_d = z_d[drafted].contiguous()
    tau = 0.5 + torch.rand(requests, device=DEV, generator=g)
    noise = -torch.log(-torch.log(torch.rand(z_d.shape, device=DEV, generator=g).clamp(1e-9, 1 - 1e-7)))
    tokens = (z_d.float() + tau.repeat_interleave(n)[:, None] * noise)[:, :VOCAB].argmax(1).to(torch.int32)
    uniforms = torch.rand(ROWS, device=DEV, generator=g)
    accepted, out = run_verify(cu, z_t, z_d, tokens, tau, uniforms, VOCAB, "bf16")
    want = verify_ref(cu, z_t, z_d, tokens, tau, uniforms, VOCAB)
    assert (accepted.tolist(), out.tolist()) == want
    ctl = K.Controller()
    assert K.tide_controller_init(ctl, K.ControllerParams(0.5, 0.9, 0.05, 4, 24, 0.75)) == 0
    for a in accepted.tolist():
        assert K.tide_controller_observe(ctl, a / n) >= 0
    assert ctl.n_seen == requests
