"""cw_attend_one against 64 bits: types, heads, head sizes, pages, lengths from none on, windows, tables with holes, what is not seen, numbers at the ends, strides,
workspaces, streams and graphs; a token behind the other with cw_cache_write, and a run of both with cw_fc4 and cw_attend."""
import math

import pytest
import torch

import paper_2006_02464_amd as cw
from attend_refs import BF16, E4M3, F16, F32, HALF_STEP, INF, NAN, Pages, assert_attention, attention, seen_causal
from operator_refs import fc4_data, fc4_weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = cw.Context(workspace_bytes=16 << 20, io_bytes=1 << 20, weight_pool_bytes=16 << 20, load_staging_bytes=1 << 20)
    yield c
    c.destroy()


@pytest.fixture(scope="module")
def space(ctx):
    w = torch.zeros(ctx.attend_one_workspace_bytes(), dtype=torch.uint8, device="cuda")
    yield w
    assert not bool(w[:cw.CW_ATTEND_COUNTERS].any())


def stream():
    return torch.cuda.current_stream()


def p_step(x, kept):
    """Of a weight in the second product: 11 bits; of bf16 two parts, the second at most 2^-7 of the first (one bf16 step of it) and off by 2^-8 of itself: 2^-15."""
    return 2.0 ** -11 if kept == E4M3 or x == F16 else 2.0 ** -15


def queries(n, heads, dim, dtype, seed, by=1.0):
    return (torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(seed)) * by).to(dtype)


def right(pool, q, scale, window=0, which=None):
    """The references of the sequences `which`, joined: (y, lse, bounds)."""
    parts = []
    for i in range(len(pool.lengths)) if which is None else which:
        n = max(0, min(pool.lengths[i], pool.table.shape[1] * pool.page))
        k, v, there = pool.read(i, 0, n)
        seen = there & ((torch.arange(n) >= pool.lengths[i] - window) if window else True)
        parts.append(attention(q[i:i + 1], k, v, scale, seen[None], p_step(q.dtype, pool.dtype)))
    return tuple(torch.cat([p[j] for p in parts]) for j in range(4))


def call(ctx, pool, q, scale, window=0, workspace=None, handle=None):
    handle = pool.cuda(ctx)[0] if handle is None else handle
    y, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    ctx.attend_one(q.cuda(), handle, pool.table.cuda(), torch.tensor(pool.lengths, dtype=torch.int32).cuda(), y, scale, window=window, lse=lse, workspace=workspace, stream=stream())
    return y.cpu(), lse.cpu()


def check(ctx, space, pool, q, scale=None, window=0, what=""):
    scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    ref = right(pool, q, scale, window)
    for workspace in (space, None):
        assert_attention(*call(ctx, pool, q, scale, window, workspace), ref, (what, workspace is not None))


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 511, 700]


@pytest.mark.parametrize("x, kept", [(F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)])
@pytest.mark.parametrize("heads, kv_heads, dim, page", [(8, 8, 64, 16), (8, 2, 128, 16), (16, 1, 128, 64), (6, 2, 80, 8), (5, 5, 16, 1), (14, 2, 256, 32), (34, 2, 96, 128), (4, 4, 240, 4), (1, 1, 32, 256),
                                                         (40, 2, 192, 2)])
def test_lengths_heads_and_sizes(ctx, space, x, kept, heads, kv_heads, dim, page):
    pool = Pages(LENGTHS, kv_heads, page, dim, kept, seed=dim).fill(dim + 1)
    check(ctx, space, pool, queries(len(LENGTHS), heads, dim, x, page))


@pytest.mark.parametrize("x, kept", [(F16, F16), (BF16, BF16), (BF16, E4M3)])
@pytest.mark.parametrize("length, sequences, heads, kv_heads, dim", [(4097, 1, 4, 4, 64), (9001, 1, 16, 2, 128), (33000, 1, 8, 1, 128), (5000, 3, 6, 3, 96), (2049, 2, 2, 2, 256)])
def test_long(ctx, space, x, kept, length, sequences, heads, kv_heads, dim):
    pool = Pages([length - 900 * i for i in range(sequences)], kv_heads, 64, dim, kept, seed=length).fill(3)
    check(ctx, space, pool, queries(sequences, heads, dim, x, 4))


@pytest.mark.parametrize("x, kept, sequences, longest, dim", [(BF16, BF16, 140, (5000, 9001, 4096), 128), (F16, E4M3, 270, (4500, 2047), 64), (F16, F16, 140, (200,), 128), (BF16, BF16, 140, (321,), 256),
                                                              (BF16, E4M3, 300, (128,), 64), (F16, F16, 300, (320, 319), 128)])
def test_more_sequences_than_run_at_once(ctx, space, x, kept, sequences, longest, dim):
    """Short ones, empty ones among them, and a few long ones: in parts, whole, or a wave each."""
    lengths = [i * 7 % 41 for i in range(sequences)]
    for i, n in enumerate(longest):
        lengths[(i * 97 + 5) % sequences] = n
    pool = Pages(lengths, 2, 16, dim, kept, seed=11).fill(9)
    check(ctx, space, pool, queries(sequences, 6, dim, x, 2))


@pytest.mark.parametrize("x, kept, lengths, heads, dim", [(BF16, BF16, [i * 37 % 900 for i in range(63)] + [3000], 6, 128), (F16, F16, [i * 37 % 900 for i in range(64)] + [3000], 6, 64),
                                                          (BF16, E4M3, [0] * 40 + [9000] + [0] * 20, 34, 128), (F16, F16, [703, 704, 705, 735, 736, 737] * 10, 2, 256), (F16, E4M3, [20000, 1], 32, 64)])
def test_parts_of_the_same_steps(ctx, space, x, kept, lengths, heads, dim):
    pool = Pages(lengths, 2, 16, dim, kept, seed=12).fill(8)
    check(ctx, space, pool, queries(len(lengths), heads, dim, x, 2))


@pytest.mark.parametrize("window", [1, 15, 16, 33, 64, 100, 512, 5000])
@pytest.mark.parametrize("kept", [BF16, E4M3])
def test_windows(ctx, space, window, kept):
    lengths = LENGTHS + [3001]
    pool = Pages(lengths, 2, 16, 64, kept, seed=2).fill(5)
    check(ctx, space, pool, queries(len(lengths), 8, 64, BF16, 6), window=window)


@pytest.mark.parametrize("kept", [F16, E4M3])
def test_tables_with_holes(ctx, space, kept):
    """Pages that are not there, whole sequences of them, numbers that are none; sequences longer than their table, lengths below zero and at the type's ends."""
    lengths = [100, 64, 500, 300, -5, -2 ** 31, 90]
    pool = Pages([max(0, n) for n in lengths], 2, 16, 64, kept, seed=2, table_pages=20).fill(5)
    pool.lengths = lengths
    pool.table[0, 2] = -1
    pool.table[0, 0] = pool.pages
    pool.table[1, :4] = -7
    pool.table[3, 5:] = 2 ** 31 - 1
    pool.table[4:6] = 0
    q = queries(len(lengths), 8, 64, F16, 6)
    check(ctx, space, pool, q)
    check(ctx, space, pool, q, window=70)
    pool.lengths[2] = 2 ** 31 - 1
    check(ctx, space, pool, q)
    check(ctx, space, pool, q, window=2 ** 31 - 1)
    pool.table = pool.table[:, :0]
    check(ctx, space, pool, q)


def test_what_is_not_seen_has_no_effect(ctx, space):
    """NaN and infinities behind the sequence's end, before the window, in the pages of others: Pages fills all of that with NaN, here with the largest numbers and infinities."""
    for kept in (F16, BF16, E4M3):
        for value in (INF, -INF, 65504.0):
            pool = Pages([37, 100, 3], 2, 16, 64, kept, seed=2)
            if kept == E4M3:
                pool.k[:], pool.v[:] = 0x7e, 0xfe
                pool.k_exp[:], pool.v_exp[:] = 254, 254
            else:
                pool.k[:], pool.v[:] = value, value
            pool.fill(5)
            q = queries(3, 8, 64, F16 if kept == E4M3 else kept, 1)
            check(ctx, space, pool, q)
            for i, n in enumerate(pool.lengths):         # and before the window
                t, page, at = pool.places(i, 0, n - 20)
                pool.k[page, :, at] = NAN if kept != E4M3 else 0x7f
                pool.v[page, :, at] = INF if kept != E4M3 else 0xff
            check(ctx, space, pool, q, window=20)


@pytest.mark.parametrize("kept", [F16, BF16])
def test_numbers_that_are_none(ctx, space, kept):
    """NaN and infinities that are seen spoil what the formula says, and nothing else: their sequence's heads, not the others'."""
    pool = Pages([70, 70, 70, 70, 70], 2, 16, 64, kept, seed=2).fill(5, loud=False)
    put = lambda x, i, t, head, d, value: x.__setitem__((pool.table[i, t // 16].long(), head, t % 16, d), value)
    put(pool.k, 0, 3, 0, 5, NAN)
    put(pool.v, 1, 69, 1, 5, NAN)
    put(pool.v, 2, 0, 1, 63, INF)
    q = queries(5, 4, 64, kept, 1)
    q[3, 2, 7] = NAN
    q[4, 1, 0] = INF
    got = [t.isnan() for t in call(ctx, pool, q, 0.125, workspace=space)]
    assert bool(got[0][0, :2].all()) and not bool(got[0][0, 2:].any())
    assert bool(got[0][1, 2:, 5].all()) and int(got[0][1].sum()) == 2
    y = call(ctx, pool, q, 0.125)[0]
    assert bool((y[2, 2:, 63] == INF).all()) and bool(y[2, :, :63].isfinite().all()) and bool(y[2, :2].isfinite().all())
    assert bool(got[0][3, 2].all()) and int(got[0][3].sum()) == 64
    assert bool(got[0][4, 1].all()) and int(got[0][4].sum()) == 64


@pytest.mark.parametrize("x, kept", [(F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)])
@pytest.mark.parametrize("what", ["equal", "one far above", "rising", "falling", "far below zero", "huge", "negative scale", "zero scale", "zero keys"])
def test_scores_of_all_kinds(ctx, space, x, kept, what):
    n, dim = 900, 64
    pool = Pages([n, 130], 1, 16, dim, kept, seed=1)
    g = torch.Generator().manual_seed(4)
    k, v = torch.randn(n, 1, dim, generator=g), torch.randn(n, 1, dim, generator=g)
    q = torch.zeros(2, 4, dim)
    q[:, :, 0] = 1.0
    q[:, :, 1:] = torch.randn(2, 4, dim - 1, generator=g) * 0.1
    t = torch.arange(n).float()[:, None]
    scale = 1.0
    if what == "equal":
        k[:] = 1.0
    elif what == "one far above":
        k[777, :, 0] = 60.0
    elif what == "rising":
        k[:, :, 0] = t * 0.2
    elif what == "falling":
        k[:, :, 0] = -t * 0.2
    elif what == "far below zero":
        k[:, :, 0] -= 3000.0
    elif what == "huge":
        k *= 200.0
    elif what == "negative scale":
        scale = -0.7
    elif what == "zero scale":
        scale = 0.0
    else:
        k[:] = 0.0
    for i in range(2):
        pool.write(i, k[:pool.lengths[i]].to(x if kept == E4M3 else kept), v[:pool.lengths[i]].to(x if kept == E4M3 else kept), pool.lengths[i])
    check(ctx, space, pool, q.to(x), scale)


@pytest.mark.parametrize("x", [F16, BF16])
def test_codes_with_exponents_of_all_sizes(ctx, space, x):
    """Values of a token 2^30 times another's: the weight that a code is multiplied with is that of its number."""
    n = 300
    pool = Pages([n, 77], 2, 16, 64, E4M3, seed=1)
    g = torch.Generator().manual_seed(4)
    by = 2.0 ** torch.randint(-14, 8, (n, 2, 1), generator=g)
    k = torch.randn(n, 2, 64, generator=g)
    v = torch.randn(n, 2, 64, generator=g) * by
    v[5:9] = 0.0
    for i in range(2):
        pool.write(i, k[:pool.lengths[i]], v[:pool.lengths[i]], pool.lengths[i])
    check(ctx, space, pool, queries(2, 6, 64, x, 2))
    pool.v_exp[:] = 127 - 20        # all small: nothing is lost
    check(ctx, space, pool, queries(2, 6, 64, BF16, 2))


@pytest.mark.parametrize("kept", [F16, E4M3])
def test_strides_and_layouts(ctx, space, kept):
    lengths = [50, 3, 170]
    pool = Pages(lengths, 2, 16, 64, kept, seed=9).fill(5)
    q = queries(3, 8, 64, F16, 3)
    ref = right(pool, q, 0.125)
    lens, table = torch.tensor(lengths, dtype=torch.int32).cuda(), torch.full((3, 40), 99, dtype=torch.int32, device="cuda")
    table[:, :pool.table.shape[1]] = pool.table.cuda()
    for layout in ("head first", "token first"):
        handle, gpu = pool.cuda(ctx, layout)
        wide = torch.full((5, 24, 64), NAN, dtype=F16, device="cuda")
        wide[1:4, 8:16] = q.cuda()
        y = torch.full((8, 5, 128), 7.0, dtype=F16, device="cuda")       # heads ahead of sequences
        out = y.transpose(0, 1)[1:4, :, 64:]
        lse = torch.zeros(3, 8, device="cuda")
        ctx.attend_one(wide[1:4, 8:16], handle, table[:, :pool.table.shape[1]], lens, out, 0.125, lse=lse, workspace=space, stream=stream())
        assert_attention(out.cpu(), lse.cpu(), ref, layout)
        assert bool((y[:, 0] == 7).all()) and bool((y[:, 4] == 7).all()) and bool((y[:, :, :64] == 7).all())
        one = torch.zeros(3, 8, 64, dtype=F16, device="cuda")            # one query for all, no lse
        ctx.attend_one(wide[1:2, 8:16].expand(3, 8, 64), handle, table[:, :pool.table.shape[1]], lens, one, 0.125, workspace=space, stream=stream())
        assert_attention(one.cpu(), None, right(pool, q[:1].expand(3, 8, 64), 0.125), layout)


@pytest.mark.parametrize("kept", [F16, E4M3])
def test_pages_far_apart(ctx, space, kept):
    far = (1 << 31) + 4096
    pool = Pages([20, 7], 2, 8, 32, kept, spare=0, seed=6).fill(8)
    size = 1 if kept == E4M3 else 2
    store = torch.empty((far * (pool.pages - 1) + (1 << 16)) * size, dtype=torch.uint8, device="cuda").view(kept)
    k, v = store.as_strided((pool.pages, 2, 8, 32), (far, 256, 32, 1)), store.as_strided((pool.pages, 2, 8, 32), (far, 256, 32, 1), storage_offset=1024)
    for to, x in ((k, pool.k), (v, pool.v)):
        to.view(torch.uint8).copy_(x) if size == 1 else to.copy_(x)
    exps = [e.cuda() if e is not None else None for e in (pool.k_exp, pool.v_exp)]
    handle = ctx.cache(k, v, k_exp=exps[0], v_exp=exps[1])
    q = queries(2, 4, 32, F16, 1)
    assert_attention(*call(ctx, pool, q, 0.2, 0, space, handle), right(pool, q, 0.2))


@pytest.mark.parametrize("size", [0, 16, 65536, 65536 + 4096, 1 << 20, 32 << 20, 100 << 20])
def test_workspaces_of_all_sizes(ctx, size):
    """More or less sharing; what lies behind the bytes that are given stays, counters are zero again."""
    pool = Pages([3000, 10, 1500], 2, 16, 128, BF16, seed=9).fill(5)
    q = queries(3, 12, 128, BF16, 3)
    store = torch.zeros(size + 4096, dtype=torch.uint8, device="cuda")
    store[size:] = 0x5a
    assert_attention(*call(ctx, pool, q, 0.08, 0, store[:size]), right(pool, q, 0.08))
    assert bool((store[size:] == 0x5a).all()) and not bool(store[:min(size, cw.CW_ATTEND_COUNTERS)].any())


@pytest.mark.parametrize("x, kept, sequences, length", [(BF16, BF16, 3, 2500), (F16, E4M3, 40, 300), (F16, F16, 300, 40)])
def test_same_bits_every_time_on_two_streams_at_once_and_replayed(ctx, x, kept, sequences, length):
    lengths = [max(1, length - 13 * i % length) for i in range(sequences)]
    pool = Pages(lengths, 2, 16, 64, kept, seed=9, table_pages=-(-length // 16) + 2).fill(5)
    handle, gpu = pool.cuda(ctx)
    table, lens, q = pool.table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), queries(sequences, 8, 64, x, 3).cuda()
    spaces = [torch.zeros(ctx.attend_one_workspace_bytes(), dtype=torch.uint8, device="cuda") for _ in range(3)]

    def go(y, lse, workspace, s):
        ctx.attend_one(q, handle, table, lens, y, 0.125, lse=lse, workspace=workspace, stream=s)
    outs = [(torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")) for _ in range(9)]
    go(*outs[8], spaces[0], stream())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(8):
        go(*outs[i], spaces[i % 2], streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o[0], outs[8][0]) and torch.equal(o[1], outs[8][1]) for o in outs)
    graphs, out = [torch.cuda.CUDAGraph() for _ in range(2)], outs[0]
    for g in graphs:                      # two graphs of one workspace, replayed one behind the other
        with torch.cuda.graph(g):
            go(*out, spaces[2], stream())
    for i in range(4):
        q.copy_(q.roll(1 + i, 2))
        lens.copy_(lens.roll(1))          # other lengths than at capture, pages that are not there among them
        table.copy_(table.roll(1, 0))
        go(*outs[1], spaces[0], stream())
        torch.cuda.synchronize()
        out[0].zero_(), out[1].zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], outs[1][0]) and torch.equal(out[1], outs[1][1])


@pytest.mark.parametrize("x, kept", [(F16, F16), (BF16, E4M3)])
def test_a_token_behind_the_other(ctx, space, x, kept):
    """Written, then attended to, on one stream and as one graph, while pages fill up; some sequences end on the way."""
    heads, kv_heads, dim, page = 6, 2, 64, 4
    pool = Pages([40, 40, 40], kv_heads, page, dim, kept, seed=3)
    pool.lengths = [0, 5, 21]
    handle, gpu = pool.cuda(ctx)
    g = torch.Generator().manual_seed(8)
    lens, table = torch.tensor(pool.lengths, dtype=torch.int32).cuda(), pool.table.cuda()
    for i, n in enumerate(pool.lengths):
        k, v = torch.randn(n, kv_heads, dim, generator=g).to(x), torch.randn(n, kv_heads, dim, generator=g).to(x)
        pool.write(i, k, v, n)
        if n:
            ctx.cache_write(k.cuda(), v.cuda(), handle, table[i:i + 1], lens[i:i + 1], first=torch.tensor([0, n], dtype=torch.int32).cuda(), stream=stream())
    q, y, lse = torch.zeros(3, heads, dim, dtype=x, device="cuda"), torch.zeros(3, heads, dim, dtype=x, device="cuda"), torch.zeros(3, heads, device="cuda")
    k, v = torch.zeros(3, kv_heads, dim, dtype=x, device="cuda"), torch.zeros(3, kv_heads, dim, dtype=x, device="cuda")
    step = torch.ones(3, dtype=torch.int32, device="cuda")

    def token():
        lens.add_(step)
        ctx.cache_write(k, v, handle, table, lens, stream=stream())
        ctx.attend_one(q, handle, table, lens, y, 0.125, lse=lse, workspace=space, stream=stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token()
    for i in range(12):
        new = [torch.randn(3, n, dim, generator=g).to(x) for n in (heads, kv_heads, kv_heads)]
        for to, t in zip((q, k, v), new):
            to.copy_(t)
        graph.replay() if i % 3 else token()
        for s in range(3):
            pool.lengths[s] += 1
            pool.write(s, new[1][s:s + 1], new[2][s:s + 1], pool.lengths[s])
        torch.cuda.synchronize()
        assert_attention(y.cpu(), lse.cpu(), right(pool, new[0], 0.125), i)


@pytest.mark.parametrize("x, kept", [(F16, F16), (BF16, BF16), (F16, E4M3)])
def test_layer_of_a_prompt_and_its_answer(ctx, space, x, kept):
    """As used: projections over 4-bit weights, the prompts' keys and values written and attended to, read back for the next part of one of them, then tokens one at a time, as one
    graph.  Against 64 bits of the numbers that the projections gave."""
    heads, kv_heads, dim, width, page = 4, 2, 64, 128, 8
    total = (heads + 2 * kv_heads) * dim
    d = fc4_data(1, width, total, 64, x, F16, True, seed=5)
    w = {n: d[n].cuda() for n in ("q", "scales", "zeros", "bias")}
    counts, history = [13, 30, 1], [0, 0, 0]
    pool = Pages([64, 64, 64], kv_heads, page, dim, kept, seed=3)
    handle, gpu = pool.cuda(ctx)
    table, lens = pool.table.cuda(), torch.zeros(3, dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(2)

    def project(rows):
        h = torch.randn(rows, width, generator=g).to(x).cuda()
        out = torch.zeros(rows, total, dtype=x, device="cuda")
        ctx.fc4(h, w["q"], w["scales"], out, 64, zeros=w["zeros"], bias=w["bias"], stream=stream())
        out = out.view(rows, heads + 2 * kv_heads, dim)
        return out, out[:, :heads], out[:, heads:heads + kv_heads], out[:, heads + kv_heads:]
    for part in (counts, [7, 2, 0]):            # whole prompts, then more of two of them behind what is there
        first = torch.tensor([0] + torch.tensor(part).cumsum(0).tolist(), dtype=torch.int32)
        lens += torch.tensor(part, dtype=torch.int32).cuda()
        pool.lengths = lens.cpu().tolist()
        _, q, k, v = project(sum(part))
        ctx.cache_write(k, v, handle, table, lens, first=first.cuda(), stream=stream())
        first_k = torch.tensor([0] + torch.tensor(pool.lengths).cumsum(0).tolist(), dtype=torch.int32)
        past = [torch.zeros(int(first_k[-1]), kv_heads, dim, dtype=x, device="cuda") for _ in range(2)]
        ctx.cache_read(handle, table, lens, past[0], past[1], first=first_k.cuda(), stream=stream())
        y, lse = torch.zeros(sum(part), heads, dim, dtype=x, device="cuda"), torch.zeros(sum(part), heads, device="cuda")
        ctx.attend(q, past[0], past[1], y, first.cuda(), 0.125, first_k=first_k.cuda(), lse=lse, stream=stream())
        torch.cuda.synchronize()
        for s in range(3):
            a, b, n = int(first[s]), int(first[s + 1]), pool.lengths[s]
            pool.write(s, k[a:b].cpu(), v[a:b].cpu(), n)
            pk, pv, _ = pool.read(s, 0, n)
            assert torch.equal(past[0][int(first_k[s]):int(first_k[s + 1])].cpu().double(), pk)
            if b > a:
                ref = attention(q[a:b].cpu(), pk, pv, 0.125, seen_causal(b - a, n), HALF_STEP[x])
                assert_attention(y[a:b].cpu(), lse[a:b].cpu(), ref, (part, s))
    hidden, out = torch.zeros(3, width, dtype=x, device="cuda"), torch.zeros(3, heads + 2 * kv_heads, dim, dtype=x, device="cuda")
    y, lse = torch.zeros(3, heads, dim, dtype=x, device="cuda"), torch.zeros(3, heads, device="cuda")

    def token():
        ctx.fc4(hidden, w["q"], w["scales"], out.view(3, total), 64, zeros=w["zeros"], bias=w["bias"], stream=stream())
        lens.add_(1)
        ctx.cache_write(out[:, heads:heads + kv_heads], out[:, heads + kv_heads:], handle, table, lens, stream=stream())
        ctx.attend_one(out[:, :heads], handle, table, lens, y, 0.125, lse=lse, workspace=space, stream=stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token()
    for i in range(5):
        hidden.copy_(torch.randn(3, width, generator=g).to(x))
        graph.replay()
        torch.cuda.synchronize()
        new = out.cpu()
        for s in range(3):
            pool.lengths[s] += 1
            pool.write(s, new[s:s + 1, heads:heads + kv_heads], new[s:s + 1, heads + kv_heads:], pool.lengths[s])
        assert_attention(y.cpu(), lse.cpu(), right(pool, new[:, :heads], 0.125), i)
