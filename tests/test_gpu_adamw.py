"""An AdamW step over a list of tensors against the definition in 64 bits: moments in 32 bits by bounds on the roundings, those in 8 bits by what their type allows,
their rounding by its mean; sizes at the borders of blocks, arrays that begin anywhere, what is not finite, graphs."""
import math

import pytest
import torch

from tests.draft_ops_util import B, DEV, HALF, TDT, Loose, gen

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS, WD = 1e-3, 0.9, 0.999, 1e-8, 0.1
F8 = torch.float8_e4m3fn


def f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def stream():
    return torch.cuda.current_stream().cuda_stream


def blocks(n):
    return (n + 255) // 256


class Tensor:
    """One tensor of a list, its arrays `off` elements behind an aligned address, with guards."""

    def __init__(self, n, param="bf16", grad="fp32", bits=8, off=0, decay=WD, seed=0, fresh=False):
        g = gen(seed)
        self.n, self.bits, self.decay, self.bf16 = n, bits, decay, param == "bf16"
        w = 0.05 * torch.randn(n, device=DEV, generator=g)
        grad_values = 1e-2 * torch.randn(n, device=DEV, generator=g) * torch.exp(1.5 * torch.randn(n, device=DEV, generator=g))
        self.a = dict(param=Loose(n, TDT[param], off, w.to(TDT[param])), grad=Loose(n, TDT[grad], off, grad_values.to(TDT[grad])))
        if self.bf16:
            self.a["master"] = Loose(n, torch.float32, off, w)
        m = torch.zeros(n, device=DEV) if fresh else 0.3 * grad_values + 1e-3 * torch.randn(n, device=DEV, generator=g)
        v = torch.zeros(n, device=DEV) if fresh else grad_values ** 2 * (0.2 + torch.rand(n, device=DEV, generator=g))
        if bits == 32:
            self.a |= dict(m=Loose(n, torch.float32, off, m), v=Loose(n, torch.float32, off, v))
        else:
            for k, x in (("m", m), ("v", v.sqrt())):
                whole = torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)
                scale = whole.abs().amax(1) / 448
                codes = (whole / scale.clamp(min=1e-30)[:, None]).clamp(-448, 448).to(F8).view(-1)[:n]
                self.a |= {k: Loose(n, F8, off, codes), k + "_scale": Loose(blocks(n), torch.float32, off, scale)}

    def row(self):
        r = {k: x.t for k, x in self.a.items()}
        return r | dict(weight_decay=self.decay)

    def state(self):
        """(w, m, v, grad) in 64 bits."""
        w = self.a["master" if self.bf16 else "param"].t.double()
        g = self.a["grad"].t.double()
        if self.bits == 32:
            return w, self.a["m"].t.double(), self.a["v"].t.double(), g
        m, r = (self.a[k].t.view(F8).double() * self.a[k + "_scale"].t.double().repeat_interleave(256)[:self.n] for k in ("m", "v"))
        return w, m, r * r, g

    def copy(self):
        c = object.__new__(Tensor)
        c.__dict__.update(self.__dict__)
        c.a = {}
        for k, x in self.a.items():
            y = object.__new__(Loose)
            y.whole, y.off = x.whole.clone(), x.off
            y.t = y.whole[x.off:x.off + x.t.numel()]
            c.a[k] = y
        return c

    def equal(self, other):
        return all(torch.equal(x.whole.view(torch.uint8), other.a[k].whole.view(torch.uint8)) for k, x in self.a.items())


def step_of(tensors, step, clip=None, seed=3, lr=LR, b1=B1, b2=B2, eps=EPS):
    B.tide_adamw(B.make_adamw_tensors([t.row() for t in tensors]), lr, b1, b2, eps, step, clip, seed, stream())


def check_step(t, before, step, clip=1.0, lr=LR, b1=B1, b2=B2, eps=EPS):
    """What tensor t holds against one step from `before` = its state()."""
    lr, b1, b2, eps, wd = f32(lr), f32(b1), f32(b2), f32(eps), f32(t.decay)
    w, m, v, g = before
    # fp32: g * clip is one rounding, a moment three more on terms that may cancel.  (8 bits: a code times its scale and the root's square are two of v's roundings.)
    gs = g * clip
    m1, m_size = b1 * m + (1 - b1) * gs, b1 * m.abs() + (1 - b1) * gs.abs()
    v1 = b2 * v + (1 - b2) * gs * gs
    m_tol, v_rel = 5 * HALF * m_size, 8 * HALF
    c1, c2 = 1 / (1 - b1 ** (step + 1)), 1 / math.sqrt(1 - b2 ** (step + 1))
    denom = v1.sqrt() * c2 + eps
    w1 = w * (1 - lr * wd) - lr * m1 * c1 / denom
    # the update: m's bound, v's halved by the root, and eight roundings (products, root, quotient, the rounded corrections and lr); the weight's own: decay, product, difference
    w_tol = abs(lr) * c1 / denom * (m_tol + m1.abs() * (v_rel / 2 + 8 * HALF)) + 3 * HALF * w.abs() + HALF * w1.abs() + 2.0 ** -149
    got = t.state()
    assert bool(((got[0] - w1).abs() <= w_tol).all()), float(((got[0] - w1).abs() - w_tol).max())
    if t.bf16:
        assert torch.equal(t.a["param"].t, t.a["master"].t.to(torch.bfloat16))
    if t.bits == 32:
        assert bool(((got[1] - m1).abs() <= m_tol + 2.0 ** -149).all()) and bool(((got[2] - v1).abs() <= v_rel * v1 + 2.0 ** -149).all())
    else:
        for key, want, tol in (("m", m1, m_tol), ("v", v1.sqrt(), v_rel * v1.sqrt())):
            scale = t.a[key + "_scale"].t.double()
            whole = torch.nn.functional.pad(want.abs(), (0, -t.n % 256)).view(-1, 256)
            top = whole.amax(1)
            slack = torch.nn.functional.pad(tol, (0, -t.n % 256)).view(-1, 256).amax(1)
            top_small = top < 2.0 ** -100
            assert bool(((scale * 448 - top).abs() <= slack + 3 * HALF * top)[~top_small].all()) and bool((scale[top_small] == 0).all())
            # the number kept is one of the two of its type around what it stands for: nearer than their distance, 2^(e - 3) with e of -6 at least
            s = scale.repeat_interleave(256)[:t.n]
            code = t.a[key].t.view(F8).double()
            x = torch.where(s > 0, want.abs() / s.clamp(min=1e-300), 0.0)
            near = tol / s.clamp(min=1e-300) + 8 * HALF * 448 * (s > 0)
            wide = torch.exp2(torch.floor(torch.log2((x + near).clamp(min=2.0 ** -6))) - 3)
            off = (code.abs() - x).abs()
            assert bool((off <= wide + near).all()), float((off - wide - near).max())
            assert bool((code.abs() <= 448).all())
            if key == "v":
                assert bool((code >= 0).all())
            else:
                sure = (want.abs() > tol) & (code != 0)
                assert torch.equal(torch.sign(code)[sure], torch.sign(want)[sure])
    for x in t.a.values():
        x.check()


SIZES = [1, 2, 7, 8, 9, 255, 256, 257, 1000, 2047, 2048, 2049, 4096 + 37, 100003]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("param,grad", [("bf16", "fp32"), ("bf16", "bf16"), ("fp32", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("off", [0, 1, 3])
def test_sizes_types_and_places(bits, param, grad, off):
    tensors = [Tensor(n, param, grad, bits, off, seed=n) for n in SIZES]
    before = [t.state() for t in tensors]
    clip = torch.tensor([0.37], device=DEV)
    step_of(tensors, 41, clip)
    for t, b in zip(tensors, before):
        check_step(t, b, 41, clip=float(clip))


@pytest.mark.parametrize("step", [0, 1, 9999, 2 ** 40])
@pytest.mark.parametrize("consts", [dict(), dict(b1=0.0), dict(b2=0.0), dict(eps=0.0), dict(eps=0.3), dict(lr=0.0), dict(lr=-0.01)], ids=str)
def test_steps_and_constants(step, consts):
    tensors = [Tensor(3001, bits=bits, seed=bits, decay=d) for bits in (8, 32) for d in (0.0, 0.3)]
    before = [t.state() for t in tensors]
    step_of(tensors, step, **consts)
    for t, b in zip(tensors, before):
        check_step(t, b, step, **consts)


def test_a_new_tensor_and_one_that_stays_zero():
    """All-zero states; a gradient of zero everywhere with eps: the weight decays and nothing else; without eps and gradient 0 / 0 is NaN as by definition."""
    for bits in (8, 32):
        t = Tensor(700, bits=bits, fresh=True)
        before = t.state()
        step_of([t], 0)
        check_step(t, before, 0)
        z = Tensor(700, bits=bits, fresh=True)
        z.a["grad"].t.zero_()
        w = z.state()[0]
        for k in range(3):
            step_of([z], k)
        want, got = w * (1 - f32(LR) * f32(WD)) ** 3, z.state()
        assert bool(((got[0] - want).abs() <= 8 * HALF * want.abs()).all()) and not got[1].any() and not got[2].any()


def test_many_tensors_mixed_in_one_list():
    """More than a launch's table holds, of both kinds and every type, empty ones between them; each as it comes out alone at the same place of a list."""
    tensors, rows = [], []
    for i in range(137):
        n = 0 if i % 11 == 5 else 1 + (i * 769) % 5000
        tensors.append(Tensor(n, "bf16" if i % 3 else "fp32", "bf16" if i % 5 == 0 else "fp32", 8 if i % 2 else 32, seed=i, decay=0.01 * i) if n else None)
        rows.append(tensors[-1].row() if n else dict(param=torch.empty(0, device=DEV), grad=torch.empty(0, device=DEV), m=torch.empty(0, device=DEV), v=torch.empty(0, device=DEV)))
    before = [t and t.state() for t in tensors]
    copies = [t and t.copy() for t in tensors]
    B.tide_adamw(B.make_adamw_tensors(rows), LR, B1, B2, EPS, 7, None, 3, stream())
    for i, (t, b) in enumerate(zip(tensors, before)):
        if t is None:
            continue
        check_step(t, b, 7)
        if i % 20 == 1:
            alone = [dict(param=torch.empty(0, device=DEV), grad=torch.empty(0, device=DEV), m=torch.empty(0, device=DEV), v=torch.empty(0, device=DEV))] * i + [copies[i].row()]
            B.tide_adamw(B.make_adamw_tensors(alone), LR, B1, B2, EPS, 7, None, 3, stream())
            assert copies[i].equal(t), i


def test_the_same_call_gives_the_same_bits_and_others_do_not():
    t = Tensor(50000, seed=1)
    runs = []
    for seed, step in ((3, 5), (3, 5), (4, 5), (3, 6)):
        c = t.copy()
        step_of([c], step, seed=seed)
        runs.append(c)
    assert runs[0].equal(runs[1])
    for other in runs[2:]:
        same = (runs[0].a["m"].t.view(torch.uint8) == other.a["m"].t.view(torch.uint8)).float().mean()
        assert 0.3 < float(same) < 0.95          # where they fell to the two sides differs
    # no two tensors and no two places share their random bits
    a, b = Tensor(50000, seed=1), Tensor(50000, seed=1)
    step_of([a, b], 5)
    assert not torch.equal(a.a["m"].t, b.a["m"].t) and not torch.equal(a.a["v"].t, b.a["v"].t)


@pytest.mark.parametrize("key", ["m", "v"])
@pytest.mark.parametrize("level", [0.9, 0.37, 0.011, 3e-4, 2.0 ** -14, 1e-6, 1e-8])
def test_rounding_is_right_in_the_mean(key, level):
    """A moment of `level` times its block's largest, 255 of 256 elements alike: the mean of what is kept is that.  Its deviation is at most half a step of the type, and the
    mean of N draws strays six times that over the root of N once in 10^9; the random bits' 16 give 2^-17 of a step beside it."""
    n = 256 * 4096
    t = Tensor(n, bits=8, fresh=True, decay=0.0)
    g = torch.full((n,), level, device=DEV)
    g[::256] = 1.0
    t.a["grad"].t.copy_(g)
    step_of([t], 0, b1=0.5, b2=0.75)
    kept = t.a[key].t.view(F8).double().view(-1, 256)[:, 1:] * t.a[key + "_scale"].t.double()[:, None]
    one = 0.5
    want, step = one * level, 2.0 ** (max(math.floor(math.log2(448 * level)), -6) - 3) * one / 448
    assert abs(float(kept.mean()) - want) <= 6 * step / 2 / math.sqrt(kept.numel()) + step * 2.0 ** -17 + 8 * HALF * one
    values = kept.unique()
    assert values.numel() <= 2 * t.a[key + "_scale"].t.unique().numel()       # the two around it and no others
    # neighbours fall independently: the correlation of N pairs strays less than six over the root of N
    up = (kept > want).double()
    if 0.02 < float(up.mean()) < 0.98:
        x = up - up.mean()
        for shift in (1, 2, 64):
            assert abs(float((x[:, shift:] * x[:, :-shift]).mean() / x.square().mean())) < 6 / math.sqrt(x[:, shift:].numel())


def test_second_moments_follow_over_many_steps():
    """Gradients of a steady size after a state of another: what a rounding to the nearest number would never leave.  The root's square is kept too large by its
    deviation: a step moves the root by delta <= (1 - beta2) r / 2 |g^2 / v - 1|, its rounding has a variance of at most delta times the type's step, r / 8, and 1 / (1 - beta2)
    steps add up: at most |g^2 / v - 1| / 16 of v, within which gradients of one size stay.  The mean of 64 K elements strays by less than a hundredth."""
    n = 65536
    t = Tensor(n, bits=8, fresh=True, decay=0.0)
    old = torch.full((n,), 0.1, device=DEV)
    old[::256] = 1.0
    t.a["grad"].t.copy_(old)
    b2 = 0.99
    for k in range(500):
        step_of([t], k, b2=b2)
    t.a["grad"].t.copy_(torch.where(old == 1.0, 1.0, 0.05))
    for k in range(500, 800):
        step_of([t], k, b2=b2)
    b = f32(b2)
    want = 0.01 * (1 - b ** 500) * b ** 300 + 0.0025 * (1 - b ** 300)
    small = t.state()[2].view(-1, 256)[:, 1:]
    assert abs(float(small.mean()) / want - 1) < 1 / 16 + 0.03      # (the way down starts at four times v: 3 / 16 of a variance that has decayed by e^-3)


def test_what_is_not_finite_stays_by_itself():
    bad = {3: float("nan"), 300: float("inf"), 515: -float("inf"), 900: 3e38, 1024: -3e38}   # (squares that overflow, too)
    for bits in (8, 32):
        t, clean = Tensor(1500, "fp32", bits=bits, seed=2), Tensor(1500, "fp32", bits=bits, seed=2)
        for i, x in bad.items():
            t.a["grad"].t[i] = x
            clean.a["grad"].t[i] = 0.0
        step_of([t], 5), step_of([clean], 5)
        fine = torch.ones(1500, dtype=torch.bool, device=DEV)
        fine[list(bad)] = False
        assert torch.equal(t.state()[0][fine], clean.state()[0][fine])
        assert bool(t.state()[0][[3, 300, 515]].isnan().all())
        if bits == 8:
            for k, where in (("m", [3, 300, 515]), ("v", list(bad))):
                code = t.a[k].t.view(F8).float()
                at = torch.zeros(1500, dtype=torch.bool, device=DEV)
                at[where] = True
                assert torch.equal(code.isnan(), at) and bool(t.a[k + "_scale"].t.isfinite().all())
            # the next step finds the others as they are
            t.a["grad"].t.nan_to_num_(0, 0, 0)
            before = t.state()
            step_of([t], 6)
            assert torch.equal(t.state()[0].isnan(), before[2].isnan() | before[1].isnan())


def test_magnitudes_at_the_ends_of_fp32():
    for size in (1e-38, 1e-31, 1e-19, 1e18):
        t = Tensor(600, bits=8, fresh=True, decay=0.0)
        t.a["grad"].t.copy_(size * torch.randn(600, device=DEV, generator=gen(1)))
        before = t.state()
        step_of([t], 0)
        for k in ("m", "v"):
            assert bool(t.a[k].t.view(F8).float().isfinite().all()) and bool(t.a[k + "_scale"].t.isfinite().all())
        assert bool(t.state()[0].isfinite().all())
        if size == 1e18:
            check_step(t, before, 0)


def test_device_schedule_gives_the_host_schedules_bits():
    a = [Tensor(5000, bits=8, seed=1), Tensor(777, bits=32, seed=2)]
    b = [t.copy() for t in a]
    lr, step, schedule = torch.tensor([LR], device=DEV), torch.tensor([10], dtype=torch.int64, device=DEV), torch.full((4,), float("nan"), device=DEV)
    listed = B.make_adamw_tensors([t.row() for t in b])
    for k in range(3):
        step_of(a, 10 + k)
        B.tide_adamw_dev(listed, lr, step, B1, B2, EPS, None, 3, schedule, stream())
    assert int(step) == 13 and all(x.equal(y) for x, y in zip(a, b))


def test_captured_and_replayed():
    """A captured step replays with the schedule of its replay; eager work and other lists between the replays."""
    a = [Tensor(5000, bits=8, seed=1), Tensor(777, bits=32, seed=2), Tensor(3, "fp32", bits=8, seed=3)]
    b, other = [t.copy() for t in a], [Tensor(900, seed=9)]
    lr, step, schedule = torch.tensor([LR], device=DEV), torch.tensor([0], dtype=torch.int64, device=DEV), torch.empty(4, device=DEV)
    clip = torch.tensor([1.0], device=DEV)
    listed = B.make_adamw_tensors([t.row() for t in b])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.tide_adamw_dev(listed, lr, step, B1, B2, EPS, clip, 3, schedule, torch.cuda.current_stream().cuda_stream)
    del listed          # the launch holds what it needs
    for k in range(5):
        for x, y in zip(a, b):
            g = torch.randn(x.n, device=DEV, generator=gen(100 + k)).to(x.a["grad"].t.dtype)
            x.a["grad"].t.copy_(g), y.a["grad"].t.copy_(g)
        lr.fill_(LR / (k + 1)), clip.fill_(0.5 + k)
        step_of(a, k, clip, lr=f32(LR / (k + 1)))
        graph.replay()
        step_of(other, k)
        torch.cuda.synchronize()
        assert all(x.equal(y) for x, y in zip(a, b)), k


def test_two_streams_at_once():
    tensors, copies = [Tensor(300000, seed=k) for k in range(2)], []
    copies = [t.copy() for t in tensors]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(4):
        for s, t in zip(streams, tensors):
            B.tide_adamw(B.make_adamw_tensors([t.row()]), LR, B1, B2, EPS, k, None, 3, s.cuda_stream)
    torch.cuda.synchronize()
    for t, c in zip(tensors, copies):
        for k in range(4):
            step_of([c], k)
        assert c.equal(t)


def test_a_tensor_beyond_32_bit_offsets():
    """4.3e9 elements: the last ones, whose offsets and random bits need more than 32 bits, against a tensor of their own."""
    n, tail = 2 ** 32 + 700, 1212           # the tail starts at a block
    w, g = torch.zeros(n, device=DEV), torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    scales = torch.zeros((2, blocks(n)), device=DEV)
    values = torch.randn(tail, device=DEV, generator=gen(4))
    w[-tail:], g[-tail:] = values, values.to(torch.bfloat16)
    small = Tensor(tail, "fp32", "bf16", 8, fresh=True)
    small.a["param"].t.copy_(values), small.a["grad"].t.copy_(values)
    before = small.state()
    B.tide_adamw(B.make_adamw_tensors([dict(param=w, grad=g, m=m, v=v, m_scale=scales[0], v_scale=scales[1], weight_decay=WD)]), LR, B1, B2, EPS, 0, None, 3, stream())
    first = n - tail
    assert first % 256 == 0
    small.a["param"].t.copy_(w[first:])
    for k, x, s in (("m", m, scales[0]), ("v", v, scales[1])):
        small.a[k].t.copy_(x[first:]), small.a[k + "_scale"].t.copy_(s[first // 256:])
    check_step(small, before, 0)
    assert not w[:first].any() and not m[:first].any()
