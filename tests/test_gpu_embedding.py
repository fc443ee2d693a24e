"""Embedding and its gradient against the definition in 64 bits: vocabularies, widths and numbers of rows at the borders of chunks, pieces and tiles, every way that
tokens repeat, arrays that begin anywhere, graphs and streams."""
import pytest
import torch

from tests.draft_ops_util import B, CODE, DEV, HALF, STEP, TDT, Loose, gen, room

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def make_ids(rows, vocab, how, seed):
    g = gen(seed)
    if how == "frequent":
        return (vocab ** torch.rand(rows, device=DEV, generator=g) - 1).to(torch.int32).clamp_(0, vocab - 1)
    if how == "one":
        return torch.full((rows,), vocab - 1, dtype=torch.int32, device=DEV)
    if how == "few":
        return torch.randint(0, min(3, vocab), (rows,), device=DEV, generator=g, dtype=torch.int32)
    if how == "ascending":
        return (torch.arange(rows, device=DEV) * vocab // max(1, rows)).to(torch.int32)
    if how == "descending":
        return make_ids(rows, vocab, "ascending", seed).flip(0)
    ids = torch.randint(0, vocab, (rows,), device=DEV, generator=g, dtype=torch.int32)
    if how == "holes":          # a third of the rows have no token: below, behind and far behind the vocabulary
        bad = torch.tensor([-1, vocab, -2 ** 31, 2 ** 31 - 1, -7], dtype=torch.int64, device=DEV).to(torch.int32)
        pick = torch.rand(rows, device=DEV, generator=g) < 0.33
        ids = torch.where(pick, bad[torch.randint(0, 5, (rows,), device=DEV, generator=g)], ids)
    if how == "none":
        ids = torch.full_like(ids, -1)
    return ids


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,d,off", [(1, 1, 1, 0), (3, 5, 7, 1), (61, 1000, 4096, 0), (130, 999, 513, 3), (1000, 37, 264, 0), (5, 9, 5121, 1)])
def test_lookup(rows, vocab, d, off, dtype):
    ids = make_ids(rows, vocab, "holes", 1)
    table = Loose(vocab * d, TDT[dtype], off, torch.randn(vocab * d, device=DEV, generator=gen(2)))
    out = Loose(rows * d, TDT[dtype], off)
    for scale in (1.0, 1.7, 0.0):
        B.tide_embed_fwd(rows, vocab, d, ids, table.t, scale, out.t, CODE[dtype], stream())
        fine = (ids >= 0) & (ids < vocab)
        s = torch.tensor(scale, dtype=torch.float32, device=DEV)
        want = torch.where(fine[:, None], table.t.view(vocab, d)[ids.clamp(0, vocab - 1).long()].float() * s, 0.0).to(TDT[dtype])   # one product, one rounding: no room
        assert torch.equal(out.t.view(rows, d), want)
        out.check()
    table.check()


@pytest.mark.parametrize("dtype,rows,d,off", [("bf16", 32768, 4096, 0), ("bf16", 33001, 4107, 1), ("fp32", 16385, 4101, 3)])
def test_lookup_of_more_than_the_last_cache(dtype, rows, d, off):
    vocab = 5000
    ids = make_ids(rows, vocab, "holes", 8)
    table = torch.randn(vocab, d, device=DEV, generator=gen(9)).to(TDT[dtype])
    out = Loose(rows * d, TDT[dtype], off)
    B.tide_embed_fwd(rows, vocab, d, ids, table, 1.7, out.t, CODE[dtype], stream())
    s = torch.tensor(1.7, dtype=torch.float32, device=DEV)
    got = out.t.view(rows, d)
    for a in range(0, rows, 4096):
        some = ids[a:a + 4096]
        fine = (some >= 0) & (some < vocab)
        want = torch.where(fine[:, None], table[some.clamp(0, vocab - 1).long()].float() * s, 0.0).to(TDT[dtype])
        assert torch.equal(got[a:a + 4096], want)
    out.check()


def gradient(ids, dy, scale, vocab, start, accumulate):
    """The definition in 64 bits, and the sums of magnitudes and the numbers of rows that bound what 32 bits may be off."""
    d = dy.shape[1]
    fine = (ids >= 0) & (ids < vocab)
    dy = dy[fine].double()
    at = ids[fine].long()
    want = torch.zeros((vocab, d), dtype=torch.float64, device=DEV).index_add_(0, at, dy) * scale
    size = torch.zeros((vocab, d), dtype=torch.float64, device=DEV).index_add_(0, at, dy.abs()) * abs(scale)
    count = torch.bincount(at, minlength=vocab)[:, None]
    if accumulate:
        want += start.double()
    return want, size, count


def check_gradient(ids, dtype, out, vocab, d, accumulate, off=0, scale=0.75, seed=5, repeat=False):
    rows = ids.numel()
    dy = Loose(rows * d, TDT[dtype], off, torch.randn(rows * d, device=DEV, generator=gen(seed)))
    fine = (ids >= 0) & (ids < vocab)
    dy.t.view(rows, d)[~fine] = float("nan")          # nothing may look at them
    start = torch.randn((vocab, d), device=DEV, generator=gen(seed + 1)).to(TDT[out])
    table = Loose(vocab * d, TDT[out], off, start if accumulate else torch.full_like(start, float("nan")))
    need = B.tide_embed_bwd_workspace_bytes(rows, vocab, d)
    ws = room(need + 256)
    args = (ids, dy.t, scale, table.t, CODE[out], accumulate, CODE[dtype], ws, need, stream())
    B.tide_embed_bwd(rows, vocab, d, *args)
    want, size, count = gradient(ids, dy.t.view(rows, d), scale, vocab, start, accumulate)
    got = table.t.view(vocab, d).double()
    # n - 1 additions, the product with the scale and the one more addition in fp32, and the rounding of the result
    tol = (count + 1) * HALF * (size + (start.double().abs() if accumulate else 0)) + STEP[out] * want.abs()
    assert bool(((got - want).abs() <= tol * 1.0001).all()), float(((got - want).abs() - tol).max())
    untouched = count[:, 0] == 0
    assert torch.equal(table.t.view(vocab, d)[untouched], start[untouched] if accumulate else torch.zeros_like(start[untouched]))
    table.check()
    assert bool((ws[need:] == 0xA5).all())
    if repeat:
        again = Loose(vocab * d, TDT[out], off, start if accumulate else start)
        B.tide_embed_bwd(rows, vocab, d, ids, dy.t, scale, again.t, CODE[out], accumulate, CODE[dtype], room(need), need, stream())
        assert torch.equal(again.t, table.t)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,out", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("rows,vocab,d", [(1, 1, 1), (2, 3, 5), (9, 4, 513), (64, 1000, 512), (65, 50, 771), (2048, 300, 264), (2049, 4000, 100)])
def test_gradient_sizes(rows, vocab, d, dtype, out, accumulate):
    check_gradient(make_ids(rows, vocab, "holes", rows), dtype, out, vocab, d, accumulate, repeat=True)


@pytest.mark.parametrize("how", ["frequent", "one", "few", "ascending", "descending", "random", "holes", "none"])
@pytest.mark.parametrize("rows", [8, 63, 2047, 6001, 40000])
def test_gradient_of_every_order(rows, how):
    check_gradient(make_ids(rows, 700, how, 3), "bf16", "fp32", 700, 96, True, repeat=rows == 40000)
    check_gradient(make_ids(rows, 700, how, 3), "fp32", "fp32", 700, 40, False)


@pytest.mark.parametrize("rows", [32768, 32769, 70001, 600000])
def test_gradient_of_many_rows(rows):
    """More than one pass of joined runs, the last run short."""
    check_gradient(make_ids(rows, 5000, "frequent", 4), "bf16", "fp32", 5000, 24, False, repeat=True)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,out,d", [("fp32", "fp32", 24), ("bf16", "bf16", 515), ("bf16", "fp32", 3)])
def test_gradient_of_tokens_over_many_pieces(dtype, out, d, accumulate):
    """Tokens whose rows reach over as many pieces of eight rows as one wave adds up, one more, as one probe sees, one more, and far more, ending at a piece's end and in it."""
    lengths = [8 * pieces + rest for pieces in (1, 15, 16, 17, 18, 32, 63, 64, 65, 66, 128, 129, 130, 257) for rest in (0, 1, 7)]
    ids = torch.repeat_interleave(torch.arange(len(lengths), device=DEV), torch.tensor(lengths, device=DEV)).to(torch.int32)
    ids = ids[torch.randperm(ids.numel(), device=DEV, generator=gen(3))]
    check_gradient(ids, dtype, out, len(lengths) + 2, d, accumulate, repeat=True)


@pytest.mark.parametrize("how", ["frequent", "one", "few", "holes"])
@pytest.mark.parametrize("rows", [127, 128, 129, 2048, 2049, 4096, 4097, 8191, 8192, 8193])
def test_gradient_at_the_borders_of_forms(rows, how):
    check_gradient(make_ids(rows, 300, how, rows), "bf16", "fp32", 300, 72, rows % 2 == 0, repeat=True)


@pytest.mark.parametrize("rows", [100, 4096, 8192])
@pytest.mark.parametrize("vocab", [2 ** 19 - 1, 2 ** 19, 2 ** 20 - 1, 2 ** 20, 2 ** 20 + 1])
def test_gradient_of_ids_that_fill_their_bits(rows, vocab):
    ids = make_ids(rows, vocab, "holes", 2)
    ids[::5] = vocab - 1
    ids[1::7] = vocab       # no token
    ids[2::7] = vocab - 2
    check_gradient(ids, "bf16", "bf16", vocab, 9, False, repeat=True)


@pytest.mark.parametrize("rows,others", [(40000, 0), (300000, 0), (300000, 777), (32768, 1)])
def test_gradient_of_one_token_in_most_rows(rows, others):
    ids = torch.full((rows,), 40, dtype=torch.int32, device=DEV)
    if others:
        ids[torch.randperm(rows, device=DEV, generator=gen(4))[:others]] = torch.randint(0, 99, (others,), device=DEV, generator=gen(6), dtype=torch.int32)
    check_gradient(ids, "bf16", "fp32", 99, 8, True, repeat=True)


@pytest.mark.parametrize("dtype,out,rows,d,off", [("bf16", "fp32", 32768, 4107, 1), ("bf16", "bf16", 32768, 4096, 0), ("fp32", "fp32", 16385, 4101, 2)])
def test_gradient_of_more_than_the_last_cache(dtype, out, rows, d, off):
    check_gradient(make_ids(rows, 3001, "holes", 1), dtype, out, 3001, d, True, off=off)


@pytest.mark.parametrize("off", [1, 2, 3, 5])
@pytest.mark.parametrize("dtype,out", [("fp32", "fp32"), ("bf16", "bf16")])
def test_gradient_of_arrays_that_begin_anywhere(off, dtype, out):
    check_gradient(make_ids(777, 90, "frequent", 6), dtype, out, 90, 1029, False, off=off)
    check_gradient(make_ids(777, 90, "frequent", 6), dtype, out, 90, 1029, True, off=off)


def test_gradient_at_the_largest_ids():
    vocab, d, rows = (1 << 21) - 1, 8, 3000
    ids = torch.randint(vocab - 20, vocab, (rows,), device=DEV, generator=gen(8), dtype=torch.int32)
    ids[::3] = vocab
    check_gradient(ids, "bf16", "bf16", vocab, d, False)


def test_table_beyond_32_bit_offsets():
    """A table of 4.3e9 elements: the last rows are as far as any."""
    vocab, d, rows = 524400, 8200, 300
    table = torch.zeros((vocab, d), dtype=torch.bfloat16, device=DEV)
    ids = torch.tensor([0, vocab - 1, vocab - 2, 262143, 262144, 524287, 524288] * 43, dtype=torch.int32, device=DEV)[:rows]
    for k in set(ids.tolist()):
        table[k] = k % 251
    out = torch.empty((rows, d), dtype=torch.bfloat16, device=DEV)
    B.tide_embed_fwd(rows, vocab, d, ids, table, 1.0, out, CODE["bf16"], stream())
    assert torch.equal(out, (ids % 251).to(torch.bfloat16)[:, None].expand(rows, d))
    need = B.tide_embed_bwd_workspace_bytes(rows, vocab, d)
    table.fill_(7)
    ones = torch.ones((rows, d), dtype=torch.bfloat16, device=DEV)
    B.tide_embed_bwd(rows, vocab, d, ids, ones, 1.0, table, CODE["bf16"], False, CODE["bf16"], room(need), need, stream())
    counts = torch.bincount(ids.long(), minlength=vocab)
    assert torch.equal(table[:, 0].float(), counts.float()) and torch.equal(table[:, -1].float(), counts.float())
    assert float(table.sum(dtype=torch.float64)) == rows * d


def test_no_rows():
    table = torch.full((50, 12), 3.0, device=DEV)
    B.tide_embed_fwd(0, 50, 12, None, None, 1.0, None, CODE["fp32"], stream())
    B.tide_embed_bwd(0, 50, 12, None, None, 1.0, table, CODE["fp32"], True, CODE["fp32"], room(1 << 16), 1 << 16, stream())
    assert bool((table == 3.0).all())
    B.tide_embed_bwd(0, 50, 12, None, None, 1.0, table, CODE["fp32"], False, CODE["fp32"], room(1 << 16), 1 << 16, stream())
    assert bool((table == 0.0).all())


def test_gradient_against_differences():
    """Of a sum of out times fixed weights: the lookup is linear in the table, so that differences are the gradient but for roundings."""
    rows, vocab, d, scale = 50, 9, 13, 1.5
    ids = make_ids(rows, vocab, "holes", 2)
    table, weights = torch.randn((vocab, d), device=DEV, generator=gen(1)), torch.randn((rows, d), device=DEV, generator=gen(2))

    def value(t):
        out = torch.empty((rows, d), device=DEV)
        B.tide_embed_fwd(rows, vocab, d, ids, t, scale, out, CODE["fp32"], stream())
        return float((out.double() * weights.double()).sum())

    dtable = torch.empty_like(table)
    need = B.tide_embed_bwd_workspace_bytes(rows, vocab, d)
    B.tide_embed_bwd(rows, vocab, d, ids, weights, scale, dtable, CODE["fp32"], False, CODE["fp32"], room(need), need, stream())
    for v, c in ((0, 0), (4, 7), (8, 12)):
        up, down = table.clone(), table.clone()
        up[v, c], down[v, c] = 1.0, -1.0       # exact numbers, two apart; each product with the scale is exact
        assert abs((value(up) - value(down)) / 2 - float(dtable[v, c])) <= (rows + 2) * HALF * float(weights.abs().sum() * scale) + 1e-12


def test_captured_and_replayed():
    """Forward and backward in a graph, replayed with other tokens and eager work between; every replay against the eager call."""
    rows, vocab, d = 5000, 800, 264
    ids, table = make_ids(rows, vocab, "frequent", 1), torch.randn((vocab, d), device=DEV).to(torch.bfloat16)
    out, dtable = torch.empty((rows, d), dtype=torch.bfloat16, device=DEV), torch.empty((vocab, d), device=DEV)
    need = B.tide_embed_bwd_workspace_bytes(rows, vocab, d)
    ws = room(need)

    def both(o, g, w):
        s = torch.cuda.current_stream().cuda_stream
        B.tide_embed_fwd(rows, vocab, d, ids, table, 2.0, o, CODE["bf16"], s)
        B.tide_embed_bwd(rows, vocab, d, ids, o, 0.5, g, CODE["fp32"], False, CODE["bf16"], w, need, s)

    both(out, dtable, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out, dtable, ws)
    for k, how in enumerate(("few", "one", "random", "holes", "frequent")):
        ids.copy_(make_ids(rows, vocab, how, 10 + k))
        dtable.fill_(float("nan"))
        graph.replay()
        o, g = torch.empty_like(out), torch.empty_like(dtable)
        both(o, g, room(need))
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(g, dtable), how


def test_two_streams_at_once():
    rows, vocab, d = 3000, 500, 520
    made, streams = [], [torch.cuda.Stream() for _ in range(2)]
    need = B.tide_embed_bwd_workspace_bytes(rows, vocab, d)
    for k in range(2):
        made.append((make_ids(rows, vocab, "frequent", k), torch.randn((rows, d), device=DEV, generator=gen(k)), torch.empty((vocab, d), device=DEV), room(need)))
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (ids, dy, g, ws) in zip(streams, made):
            B.tide_embed_bwd(rows, vocab, d, ids, dy, 1.0, g, CODE["fp32"], False, CODE["fp32"], ws, need, s.cuda_stream)
    torch.cuda.synchronize()
    for ids, dy, g, ws in made:
        alone = torch.empty_like(g)
        B.tide_embed_bwd(rows, vocab, d, ids, dy, 1.0, alone, CODE["fp32"], False, CODE["fp32"], room(need), need, stream())
        assert torch.equal(alone, g)
