"""Verification of drafted tokens against the definition in 64 bits on the host: every token has to be the same one.  (The library's exponentials are off by 1e-12 at most, so that
one number in some millions could fall between its border and the definition's; the seeds are fixed.)"""
import math

import pytest
import torch

from tests.draft_ops_util import B, CODE, DEV, TDT, gen, room, run_verify, verify_ref

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def floats(*x):
    return torch.tensor(x, dtype=torch.float32, device=DEV)


def batch(lens, vocab, dtype, seed, extra=0, spread=3.0, near=0.7, behind=0):
    """Logits (columns behind the vocabulary hold NaN), drafts near the target's, tokens drawn from them, numbers."""
    g = gen(seed)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n + 1)
    rows, ld = cu[-1] + behind, (vocab + 7) // 8 * 8 + extra
    drafted = rows - len(lens)
    target = torch.full((rows, ld), NAN, device=DEV, dtype=TDT[dtype])
    target[:, :vocab] = spread * torch.randn((rows, vocab), device=DEV, generator=g)
    draft = torch.full((max(1, drafted), ld), NAN, device=DEV, dtype=TDT[dtype])
    at = torch.tensor([cu[b] + i for b, n in enumerate(lens) for i in range(n)], dtype=torch.long, device=DEV)
    temperature = 0.4 + torch.rand(len(lens), device=DEV, generator=g)
    tokens = torch.zeros(drafted, dtype=torch.int32, device=DEV)
    if len(at):
        draft[:len(at), :vocab] = target[at, :vocab].float() + near * torch.randn((len(at), vocab), device=DEV, generator=g)
        tau = temperature.repeat_interleave(torch.tensor(lens, device=DEV))[:, None]
        noise = -torch.log(-torch.log(torch.rand((len(at), vocab), device=DEV, generator=g).clamp(1e-9, 1 - 1e-7)))
        tokens[:len(at)] = (draft[:len(at), :vocab].float() + tau * noise).argmax(1).to(torch.int32)
    return ints(*cu), target, draft[:drafted], tokens, temperature, torch.rand(rows, device=DEV, generator=g)


def check(cu, target, draft, tokens, temperature, uniforms, vocab, dtype):
    accepted, out = run_verify(cu, target, draft, tokens, temperature, uniforms, vocab, dtype)
    want_accepted, want = verify_ref(cu, target, draft, tokens, temperature, uniforms, vocab)
    assert accepted.tolist() == want_accepted
    n = int(cu[-1])
    assert out[:n].tolist() == want
    assert bool((out[n:] == 77).all())          # rows behind the last request
    return want_accepted


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 2047, 2048, 2049, 4097, 8192, 8193, 32001, 128256])
def test_vocabularies(vocab, dtype):
    for how, lens in (("ragged", [3, 0, 4, 1, 0, 2, 7]), ("one", [3]), ("bare", [0])):
        cu, target, draft, tokens, temperature, uniforms = batch(lens, vocab, dtype, vocab + len(lens), extra=16)
        check(cu, target, draft, tokens, temperature, uniforms, vocab, dtype)
        check(cu, target, None, tokens, temperature, uniforms, vocab, dtype)
        check(cu, target, draft, tokens, None, uniforms, vocab, dtype)
        temperature[::2] = 0.0
        check(cu, target, draft, tokens, temperature, uniforms, vocab, dtype)


@pytest.mark.parametrize("lens", [[1] * 300, [8, 0, 3] * 70, [40, 1, 130], [5] * 1100], ids=["300", "210", "long", "1100"])
def test_numbers_of_requests_and_drafts(lens):
    for dtype, vocab, near in (("bf16", 1003, 0.3), ("fp32", 264, 0.05)):
        data = batch(lens, vocab, dtype, 5, near=near)
        got = check(*data, vocab, dtype)
        assert max(got) > 0 and any(a < n for a, n in zip(got, lens))


@pytest.mark.parametrize("requests", [257, 5000, 20000])
def test_many_requests(requests):
    """More than are looked through at once for the one that a row belongs to."""
    lens = [(b * b + b // 7) % 4 for b in range(requests)]
    check(*batch(lens, 40, "fp32", requests, near=0.5), 40, "fp32")


def test_large_batches_take_wider_parts():
    """Rows enough for wider parts, for sums in 32 bits first, and for parts of 16384 and 32768 columns; requests without sampling, without a distribution and at
    temperatures for which 32 bits are no good among them; a draft and none."""
    for requests, vocab, dtype in ((60, 20003, "bf16"), (200, 20003, "fp32"), (40, 128256, "bf16"), (70, 40001, "bf16")):
        cu, target, draft, tokens, temperature, uniforms = batch([4] * requests, vocab, dtype, 9, near=0.4)
        check(cu, target, draft, tokens, temperature, uniforms, vocab, dtype)
        temperature[::5] = 0.0
        temperature[1], temperature[6], temperature[7], temperature[8] = 1e-32, 1e32, NAN, -1.0
        target[5 * 11 + 1, 17], target[5 * 12, vocab - 1], draft[4 * 13 + 2, 8] = NAN, INF, NAN
        target[5 * 14, :vocab] = -INF
        target[5 * 16:5 * 18, 5:vocab:2] = -INF
        check(cu, target, draft, tokens, temperature, uniforms, vocab, dtype)
        check(cu, target, None, tokens, temperature, uniforms, vocab, dtype)


def test_rows_behind_the_last_request_are_left_alone():
    cu, target, draft, tokens, temperature, uniforms = batch([2, 3], 500, "bf16", 3, behind=4)
    tokens[-4:] = 2 ** 31 - 1
    uniforms[-4:] = NAN
    check(cu, target, draft, tokens, temperature, uniforms, 500, "bf16")


@pytest.mark.parametrize("vocab,half", [(1024, 512), (2048, 256), (16384, 8192), (131072, 65536)])
def test_acceptance_at_its_border(vocab, half):
    """Both distributions are even, the draft's over fewer columns: p / q is half / vocab exactly, and a number of that is not below it."""
    ratio = half / vocab
    below = float(torch.nextafter(floats(ratio), floats(0.0)))
    for u, takes in ((ratio, 0), (below, 1)):
        target, draft = torch.zeros((2, vocab), device=DEV), torch.full((1, vocab), -INF, device=DEV)
        draft[0, -half:] = 0
        accepted, out = run_verify(ints(0, 2), target, draft, ints(vocab - 3), floats(0.7), floats(u, 0.0), vocab, "fp32")
        assert int(accepted) == takes
        # refused: the columns that the draft has none of keep all of their weight, the others nothing; the number 0 takes the first
        assert out.tolist() == ([vocab - 3, 0] if takes else [0, -1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_borders_in_batches_whose_sums_are_made_in_32_bits_first(dtype):
    """120 requests over 65536 columns: more than are summed in 64 bits at once.  Each request meets its border at several positions: even distributions, the draft's over half, a quarter, an
    eighth of the columns, and numbers at the quotient, the next below and the next above."""
    vocab, n = 65536, 3
    steps = [0.5, 0.25, 0.125]
    cu = ints(*range(0, 4 * 120 + 1, 4))
    target = torch.full((480, vocab), 1.25, device=DEV, dtype=TDT[dtype])
    draft = torch.full((360, vocab), -INF, device=DEV, dtype=TDT[dtype])
    numbers, want, tokens = [], [], []
    for b in range(120):
        j = n
        for i in range(n):
            ratio = steps[(b + i) % 3]
            draft[3 * b + i, :int(vocab * ratio)] = -2.5
            kind = (b // 3 + 2 * i * (b % 5)) % 3
            u = [float(torch.nextafter(torch.tensor(ratio), torch.tensor(0.0))), ratio, float(torch.nextafter(torch.tensor(ratio), torch.tensor(1.0)))][kind]
            j = min(j, i) if kind else j
            numbers.append(u), tokens.append((977 * b + i) % int(vocab * ratio))
        k = (613 * b) % 1024           # the emitted token at a border too
        numbers.append(k / 1024)
        if j == n:
            token = 64 * k
        else:                          # p - q is left where the draft has nothing
            ratio = steps[(b + j) % 3]
            first, left = int(vocab * ratio), vocab - int(vocab * ratio)
            token = first + math.floor(k / 1024 * left)
            if (k * left) % 1024:      # (between two columns there is no border)
                token = first + k * left // 1024
        want += tokens[3 * b:3 * b + j] + [token] + [-1] * (n - j)
    accepted, out = run_verify(cu, target, draft, ints(*tokens), None, floats(*numbers), vocab, dtype)
    assert out.tolist() == want
    assert 0 < int(accepted.sum()) < 360


@pytest.mark.parametrize("vocab", [1024, 16384, 131072])
def test_the_emitted_token_at_its_borders(vocab):
    """An even distribution cumulates to k / vocab exactly; a number of k / vocab belongs to column k, the one below it to k - 1."""
    ks = [0, 1, 2, 7, 8, 255, 256, 511, 512, 1000, vocab // 2, vocab - 1]
    numbers, want = [], []
    for k in ks:
        numbers.append(k / vocab), want.append(k)
        if k:
            numbers.append(float(torch.nextafter(floats(k / vocab), floats(0.0)))), want.append(k - 1)
    target = torch.zeros((len(numbers), vocab), device=DEV, dtype=torch.bfloat16)
    accepted, out = run_verify(ints(*range(len(numbers) + 1)), target, None, ints(), floats(*([0.3] * len(numbers))), floats(*numbers), vocab, "bf16")
    assert out.tolist() == want and not accepted.any()
    # every second column masked: half as many, the same borders
    target[:, ::2] = -INF
    numbers = [min(2 * k / vocab, 1 - 2 ** -24) for k in range(4)]
    accepted, out = run_verify(ints(0, 1, 2, 3, 4), target[:4], None, ints(), None, floats(*numbers), vocab, "bf16")
    assert out.tolist() == [1, 3, 5, 7]


def test_numbers_outside_of_their_range():
    """1 and more, NaN, below 0: the emitted token is one with weight (the last, the first); acceptance follows its comparison."""
    vocab = 3000
    target = torch.full((5, vocab), -INF, device=DEV)
    target[:, 100:200] = 1.0
    for u, want in ((1.0, 199), (7.0, 199), (INF, 199), (NAN, 100), (-1.0, 100), (0.0, 100)):
        _, out = run_verify(ints(0, 1), target[:1], None, ints(), None, floats(u), vocab, "fp32")
        assert out.tolist() == [want], u
    # a number of 1 refuses what both agree on; nothing is left of p - q, and the target's own distribution stands in
    accepted, out = run_verify(ints(0, 2), target[:2], target[:1].clone(), ints(150), None, floats(1.0, 0.5), vocab, "fp32")
    assert accepted.tolist() == [0] and out.tolist() == [150, -1]
    accepted, out = run_verify(ints(0, 2), target[:2], target[:1].clone(), ints(150), None, floats(NAN, 0.995), vocab, "fp32")
    assert accepted.tolist() == [0] and out.tolist() == [199, -1]
    # also where probabilities are no round numbers, and in a batch
    for lens in ([1] * 3, [1] * 200):
        cu, target, _, tokens, temperature, uniforms = batch(lens, 32001, "bf16", 41)
        draft = target[cu[:-1].long()].contiguous()
        uniforms[::2] = 1.0
        check(cu, target, draft, tokens, temperature, uniforms, 32001, "bf16")


def test_tokens_that_are_none_end_the_draft():
    vocab = 700
    cu, target, draft, tokens, temperature, uniforms = batch([4, 4, 4, 4], vocab, "bf16", 11, near=0.01)
    tokens[1], tokens[4], tokens[10], tokens[15] = -1, vocab, 2 ** 31 - 1, -2 ** 31
    got = check(cu, target, draft, tokens, temperature, uniforms, vocab, "bf16")
    assert got[0] <= 1 and got[1] == 0 and got[2] <= 2 and got[3] <= 3
    temperature.zero_()
    check(cu, target, draft, tokens, temperature, uniforms, vocab, "bf16")


@pytest.mark.parametrize("tau", [0.0, 0.8])
def test_rows_without_a_distribution(tau):
    """NaN anywhere, +inf, nothing but -inf: in a target row the token is refused and -1 emitted, in a draft row the token is refused and p stands alone."""
    vocab = 9001
    lens = [3] * 8
    for where in (0, 4095, 9000):
        cu, target, draft, tokens, _, uniforms = batch(lens, vocab, "fp32", 13, near=0.0)     # the draft agrees: what is whole is accepted
        temperature = torch.full((8,), tau, device=DEV)
        if tau == 0.0:
            tokens = target[[4 * b + i for b in range(8) for i in range(3)], :vocab].argmax(1).to(torch.int32)
        target[0, where] = NAN
        target[4 + 1, where] = INF
        target[8 + 2, :vocab] = -INF
        target[12 + 3, where] = NAN                # the row behind all drafts
        draft[12, where] = NAN                     # request 4
        draft[16, where] = INF
        draft[20, :vocab] = -INF
        accepted, out = run_verify(cu, target, draft, tokens, temperature, uniforms, vocab, "fp32")
        want = verify_ref(cu, target, draft, tokens, temperature, uniforms, vocab)
        assert (accepted.tolist(), out.tolist()) == want
        assert accepted.tolist() == ([0, 1, 2, 3, 3, 3, 3, 3] if tau == 0.0 else [0, 1, 2, 3, 0, 1, 2, 3])
        for b in range(4):
            assert int(out[4 * b + int(accepted[b])]) == -1
    for tau in (-1.0, NAN, INF, -0.1):
        accepted, out = run_verify(ints(0, 2, 3), torch.zeros((3, 16), device=DEV), None, ints(3), floats(tau, 1.0), floats(0.1, 0.1, 0.1), 16, "fp32")
        assert accepted.tolist() == [0, 0] and out.tolist() == [-1, -1, 1]


def test_masked_columns_and_extreme_logits():
    """-inf and the type's lowest value as masks, logits of 1e30, temperatures of 1e-6 and 1e6, one column that is all."""
    for dtype in ("bf16", "fp32"):
        vocab, lens = 5003, [2, 1, 3, 0]
        for mask in (-INF, torch.finfo(TDT[dtype]).min):
            cu, target, draft, tokens, temperature, uniforms = batch(lens, vocab, dtype, 17)
            hide = torch.rand((target.shape[0], vocab), device=DEV, generator=gen(1)) < 0.9
            target[:, :vocab] = torch.where(hide, mask, target[:, :vocab])
            check(cu, target, draft, tokens, temperature, uniforms, vocab, dtype)
            draft[:, :vocab] = torch.where(hide[:draft.shape[0]], mask, draft[:, :vocab])
            check(cu, target, draft, tokens, temperature, uniforms, vocab, dtype)
        for scale, tau in ((1e30, 1.0), (1e30, 1e30), (1.0, 1e-6), (1.0, 1e6), (1.0, 1e-30), (100.0, 1e-2), (1e-30, 1.0)):
            cu, target, draft, tokens, temperature, uniforms = batch(lens, vocab, dtype, 19)
            target, draft = (target.float() * scale).to(TDT[dtype]), (draft.float() * scale).to(TDT[dtype])
            temperature.fill_(tau)
            check(cu, target, draft, tokens, temperature, uniforms, vocab, dtype)


def test_ties_of_the_largest_logit_go_to_the_first():
    vocab = 40000
    target = torch.zeros((3, vocab), device=DEV, dtype=torch.bfloat16)
    target[0, [39999, 8191, 8192, 20000]] = 2.0
    target[1, 0] = -0.0
    target[2, 5:] = 1.0
    accepted, out = run_verify(ints(0, 1, 2, 3), target, None, ints(), floats(0.0, 0.0, 0.0), floats(0.9, 0.9, 0.9), vocab, "bf16")
    assert out.tolist() == [8191, 0, 5]


def test_emitted_tokens_are_distributed_as_the_target():
    """Whatever the draft: of 60000 requests the first token's frequencies, each within six deviations of the target's probability."""
    vocab, n = 11, 60000
    g = gen(21)
    z, y = 1.5 * torch.randn(vocab, device=DEV, generator=g), 1.5 * torch.randn(vocab, device=DEV, generator=g)
    ld = 16
    target, draft = torch.zeros((2 * n, ld), device=DEV), torch.zeros((n, ld), device=DEV)
    target[:, :vocab], draft[:, :vocab] = z, y
    tau = 0.9
    noise = -torch.log(-torch.log(torch.rand((n, vocab), device=DEV, generator=g, dtype=torch.float64)))
    drawn = (y.double() + tau * noise).argmax(1).to(torch.int32)
    cu, uniforms = torch.arange(0, 2 * n + 1, 2, dtype=torch.int32, device=DEV), torch.rand(2 * n, device=DEV, generator=g)
    p = torch.softmax(z.double() / tau, 0)
    for d, x in ((draft, drawn), (None, torch.full_like(drawn, 4)), (None, drawn)):
        _, out = run_verify(cu, target, d, x, torch.full((n,), tau, device=DEV), uniforms, vocab, "fp32")
        share = torch.bincount(out[::2].long(), minlength=vocab).double() / n
        if d is not None or len(x.unique()) == 1:
            assert bool(((share - p).abs() <= 6 * (p * (1 - p) / n).sqrt()).all()), (share, p)


def test_offsets_out_of_order_stay_inside():
    """Meaningless numbers, but nothing outside of the arrays is written, and a request whose rows no other claims comes out right."""
    vocab, rows = 300, 12
    cu, target, draft, tokens, temperature, uniforms = batch([3, 3, 3], vocab, "bf16", 23)
    for bad in ([0, 4, 2, 12], [0, 4, 100, 12], [-5, 4, 8, 12], [0, 4, 8, 2 ** 31 - 1], [0, 4, 4, 12], [12, 8, 4, 0], [-2 ** 31, -1, -1, -1], [7, 7, 7, 7]):
        whole = torch.full((rows + 64,), 77, dtype=torch.int32, device=DEV)
        acc = torch.full((3 + 64,), 77, dtype=torch.int32, device=DEV)
        need = B.tide_verify_workspace_bytes(rows, 3, vocab)
        ws = room(need + 256)
        B.tide_verify_drafts(rows, 3, vocab, ints(*bad), target, target.shape[1], draft, draft.shape[1], tokens, temperature, uniforms, acc[32:35], whole[32:32 + rows], CODE["bf16"],
                             ws, need, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert bool((whole[:32] == 77).all()) and bool((whole[32 + rows:] == 77).all()) and bool((acc[:32] == 77).all()) and bool((acc[35:] == 77).all())
        assert bool((ws[need:] == 0xA5).all())
        if bad[:2] == [0, 4] and min(bad[1:]) >= 4:      # (in [0, 4, 2, 12] the last request owns rows from 2 on, and writes there too)
            want = verify_ref(cu[:2], target, draft, tokens, temperature, uniforms, vocab)
            assert int(acc[32]) == want[0][0] and whole[32:36].tolist() == want[1]


def test_captured_and_replayed_with_a_workspace_that_others_use():
    vocab = 32001
    data = batch([4, 2, 0, 5], vocab, "bf16", 29)
    cu, target, draft, tokens, temperature, uniforms = data
    rows = target.shape[0]
    need = B.tide_verify_workspace_bytes(rows, 4, vocab)
    ws = room(need)
    accepted, out = torch.empty(4, dtype=torch.int32, device=DEV), torch.empty(rows, dtype=torch.int32, device=DEV)

    def call():
        B.tide_verify_drafts(rows, 4, vocab, cu, target, target.shape[1], draft, draft.shape[1], tokens, temperature, uniforms, accepted, out, CODE["bf16"], ws, need,
                             torch.cuda.current_stream().cuda_stream)

    call()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            call()
    for k in range(6):
        fresh = batch([4, 2, 0, 5], vocab, "bf16", 100 + k)
        for old, new in zip(data[1:], fresh[1:]):
            old.copy_(new)
        if k % 2:
            ws.fill_(0xFF)
        out.fill_(77)
        graphs[k % 2].replay()
        run_verify(*batch([1, 1], 500, "fp32", k), 500, "fp32")
        torch.cuda.synchronize()
        assert (accepted.tolist(), out.tolist()) == verify_ref(*data, vocab), k


def test_two_streams_at_once():
    vocab, made, streams = 50001, [], [torch.cuda.Stream() for _ in range(2)]
    for k in range(2):
        data = batch([3] * 6, vocab, "bf16", 31 + k)
        rows = data[1].shape[0]
        need = B.tide_verify_workspace_bytes(rows, 6, vocab)
        made.append((data, room(need), need, torch.empty(6, dtype=torch.int32, device=DEV), torch.empty(rows, dtype=torch.int32, device=DEV)))
    torch.cuda.synchronize()
    for _ in range(10):
        for s, ((cu, target, draft, tokens, temperature, uniforms), ws, need, accepted, out) in zip(streams, made):
            B.tide_verify_drafts(out.numel(), 6, vocab, cu, target, target.shape[1], draft, draft.shape[1], tokens, temperature, uniforms, accepted, out, CODE["bf16"], ws, need, s.cuda_stream)
    torch.cuda.synchronize()
    for data, _, _, accepted, out in made:
        assert (accepted.tolist(), out.tolist()) == verify_ref(*data, vocab)


def test_logits_beyond_32_bit_offsets():
    """Rows of a stride of 2^28 columns: the last ones lie more than 2^32 bytes and elements away."""
    vocab, ld = 1000, 1 << 28
    cu, small, draft, tokens, temperature, uniforms = batch([5, 4, 5], vocab, "bf16", 37)
    rows = small.shape[0]
    target = torch.zeros((rows, ld), dtype=torch.bfloat16, device=DEV)
    target[:, :vocab] = small[:, :vocab]
    assert rows * ld > 2 ** 32
    accepted, out = run_verify(cu, target, draft, tokens, temperature, uniforms, vocab, "bf16")
    assert (accepted.tolist(), out.tolist()) == verify_ref(cu, small, draft, tokens, temperature, uniforms, vocab)


def test_a_vocabulary_of_many_parts():
    """2^24 columns and a border in the last of them."""
    vocab = (1 << 24) - 3
    target = torch.full((2, 1 << 24), -INF, device=DEV)
    target[0, 5], target[0, vocab - 1] = 0.0, math.log(3.0)
    target[1, vocab - 1] = 0.0
    for u, want in ((0.2, 5), (0.26, vocab - 1)):
        accepted, out = run_verify(ints(0, 1, 2), target, None, ints(), None, floats(u, u), vocab, "fp32")
        assert out.tolist() == [want, vocab - 1]
