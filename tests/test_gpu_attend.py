"""cw_attend against 64 bits: types, heads, head sizes, packed lengths from none on, keys ahead of the queries or fewer than them, windows, what is not seen, numbers at the ends,
strides, far rows, streams and graphs."""
import math

import pytest
import torch

import paper_2006_02464_amd as cw
from attend_refs import BF16, F16, F32, HALF_STEP, INF, NAN, assert_attention, attention, seen_causal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = cw.Context(workspace_bytes=16 << 20, io_bytes=1 << 20, weight_pool_bytes=16 << 20, load_staging_bytes=1 << 20)
    yield c
    c.destroy()


def stream():
    return torch.cuda.current_stream()


def starts(counts, begin=0):
    return torch.tensor([begin] + (torch.tensor(counts).cumsum(0) + begin).tolist(), dtype=torch.int32)


def data(counts, counts_k, heads, kv_heads, dim, dtype, seed=0, loud=True):
    g = torch.Generator().manual_seed(seed)
    by = 1.0 + 9.0 * (torch.rand(kv_heads, dim, generator=g) < 0.03) if loud else 1.0
    make = lambda n, h, by: (torch.randn(n, h, dim, generator=g) * by).to(dtype)
    return make(sum(counts), heads, 1.0), make(sum(counts_k), kv_heads, by), make(sum(counts_k), kv_heads, 1.0)


def right(q, k, v, counts, counts_k, scale, causal=True, window=0):
    parts, a, b = [], 0, 0
    for n, m in zip(counts, counts_k):
        if n:
            parts.append(attention(q[a:a + n], k[b:b + m], v[b:b + m], scale, seen_causal(n, m, causal, window), HALF_STEP[q.dtype]))
        a, b = a + n, b + m
    return tuple(torch.cat([p[j] for p in parts]) for j in range(4))


def check(ctx, q, k, v, counts, counts_k, scale=None, causal=True, window=0, what=""):
    scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    y, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    same = list(counts) == list(counts_k)
    ctx.attend(q.cuda(), k.cuda(), v.cuda(), y, starts(counts).cuda(), scale, first_k=None if same else starts(counts_k).cuda(), causal=causal, window=window, lse=lse, stream=stream())
    assert_attention(y.cpu(), lse.cpu(), right(q, k, v, counts, counts_k, scale, causal, window), what)


COUNTS = [1, 2, 0, 31, 32, 33, 64, 1, 65, 127, 130, 0, 5]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads, kv_heads, dim", [(2, 2, 64), (4, 1, 128), (3, 3, 80), (2, 1, 256), (7, 7, 16), (4, 2, 96), (1, 1, 32), (2, 2, 240), (6, 2, 192), (2, 2, 112)])
def test_packed_lengths_heads_and_sizes(ctx, dtype, causal, heads, kv_heads, dim):
    q, k, v = data(COUNTS, COUNTS, heads, kv_heads, dim, dtype, dim)
    check(ctx, q, k, v, COUNTS, COUNTS, causal=causal)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("length", [255, 256, 257, 700, 1025])
@pytest.mark.parametrize("dim", [64, 128])
def test_one_prompt(ctx, dtype, length, dim):
    q, k, v = data([length], [length], 4, 2, dim, dtype, length)
    check(ctx, q, k, v, [length], [length])
    check(ctx, q, k, v, [length], [length], causal=False)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 96])
def test_other_numbers_of_keys_than_of_queries(ctx, dtype, causal, dim):
    """Parts behind their histories; fewer keys than queries, whose first rows see nothing; no keys."""
    counts, counts_k = [1, 40, 130, 3, 70, 5, 0, 64, 200], [500, 41, 300, 0, 20, 5, 10, 193, 100]
    q, k, v = data(counts, counts_k, 4, 2, dim, dtype, 3)
    check(ctx, q, k, v, counts, counts_k, causal=causal)


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 100, 129, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("dim", [64, 128])
def test_windows(ctx, window, dim):
    counts, counts_k = [1, 40, 130, 300, 70, 0, 64], [500, 41, 300, 300, 20, 10, 193]
    q, k, v = data(counts, counts_k, 4, 2, dim, BF16, 3)
    check(ctx, q, k, v, counts, counts_k, window=window)


def test_many_sequences(ctx):
    for n in (64, 65, 1000, 4097):
        counts = [i * 7 % 5 for i in range(n)]
        counts_k = [i * 3 % 4 + c for i, c in enumerate(counts)]
        q, k, v = data(counts, counts_k, 2, 1, 32, F16, n)
        y, lse = torch.full(q.shape, 7.0, dtype=F16, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
        ctx.attend(q.cuda(), k.cuda(), v.cuda(), y, starts(counts).cuda(), 0.2, first_k=starts(counts_k).cuda(), lse=lse, stream=stream())
        ref = right(q, k, v, counts, counts_k, 0.2)
        assert_attention(y.cpu(), lse.cpu(), ref, n)


def test_rows_that_belong_to_no_sequence_stay(ctx):
    counts = [20, 0, 150]
    q, k, v = data(counts, counts, 4, 2, 64, F16, 3)
    pad = lambda t: torch.cat([torch.full((5, *t.shape[1:]), NAN, dtype=t.dtype), t, torch.full((300, *t.shape[1:]), NAN, dtype=t.dtype)])
    y, lse = torch.full((475, 4, 64), 7.0, dtype=F16, device="cuda"), torch.full((475, 4), 7.0, device="cuda")
    ctx.attend(pad(q).cuda(), pad(k).cuda(), pad(v).cuda(), y, starts(counts, 5).cuda(), 0.125, lse=lse, stream=stream())
    assert_attention(y[5:175].cpu(), lse[5:175].cpu(), right(q, k, v, counts, counts, 0.125))
    for t in (y, lse):
        assert bool((t[:5] == 7).all()) and bool((t[175:] == 7).all())


def test_starts_that_leave_the_rows(ctx):
    """Rows that are none are left out: nothing is read or written outside the tensors (their neighbours stay)."""
    q, k, v = data([100], [100], 2, 1, 64, F16, 3)
    store = torch.full((300, 2, 64), 7.0, dtype=F16, device="cuda")
    y = store[100:200]
    for first, first_k in (([0, 100, 500], [0, 100, 200]), ([0, 50, 2 ** 31 - 1], None), ([-50, 20, 100], None), ([0, 100], [-20, 90]), ([0, 100], [50, 2 ** 31 - 1]), ([60, 20, 100], None),
                           ([0, 100], [90, 10]), ([-2 ** 31, 2 ** 31 - 1], None), ([0, 100], [-2 ** 31, 2 ** 31 - 1])):
        lse = torch.full((100, 2), 7.0, device="cuda")
        ctx.attend(q.cuda(), k.cuda(), v.cuda(), y, torch.tensor(first, dtype=torch.int32).cuda(), 0.125, first_k=None if first_k is None else torch.tensor(first_k, dtype=torch.int32).cuda(),
                   lse=lse, stream=stream())
        torch.cuda.synchronize()
        assert bool((store[:100] == 7).all()) and bool((store[200:] == 7).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_is_not_seen_has_no_effect(ctx, dtype, value, dim):
    """Keys and values behind a query in its own tile, before its window, of the neighbours: queries that do not see them are as if they were numbers."""
    counts = [70, 200, 40]
    q, k, v = data(counts, counts, 2, 2, dim, dtype, 7, loud=False)
    k[75 + 90:75 + 92, 1], v[70 + 100, 0, 3], v[70 + 130, 0, :], v[70 + 131, 1, 7] = value, value, value, value
    k[269, 0, 0], v[269, 1] = value, value
    k[0, 0, 0], v[69, 0, 1] = value, value
    for causal, window in ((True, 0), (True, 37), (True, 3)):
        y, lse = torch.zeros(q.shape, dtype=dtype, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
        ctx.attend(q.cuda(), k.cuda(), v.cuda(), y, starts(counts).cuda(), 0.1, window=window, lse=lse, stream=stream())
        ry, rl, oy, ol = right(q, k, v, counts, counts, 0.1, causal, window)
        y, lse = y.cpu(), lse.cpu()
        clean = ry.isfinite() & rl.isfinite()[..., None]      # rows that see a key of +-inf or NaN may hold what the formula leaves open
        assert float(clean.double().mean()) > 0.2
        bound = oy + HALF_STEP[dtype] * (ry.abs() + oy) + 1e-7
        assert bool(((y.double() - ry).abs() <= bound)[clean].all()), (window, ((y.double() - ry).abs() / bound)[clean].max())
        spoiled = ry.isnan() & rl.isfinite()[..., None]
        assert bool(y.isnan()[spoiled].all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("what", ["equal", "one far above", "rising", "falling", "far below zero", "huge", "negative scale", "zero scale", "zero keys"])
def test_scores_of_all_kinds(ctx, dtype, what):
    n, dim = 520, 64
    q, k, v = data([n], [n], 2, 1, dim, F32, 4, loud=False)
    q *= 0.1
    q[:, :, 0] = 1.0
    t = torch.arange(n).float()[:, None]
    scale = 1.0
    if what == "equal":
        k[:] = 1.0
    elif what == "one far above":
        k[300, :, 0] = 60.0
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
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    check(ctx, q, k, v, [n], [n], scale, True)
    check(ctx, q, k, v, [n], [n], scale, False)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_strides(ctx, dtype):
    """Parts of a projection's result; heads ahead of tokens; one key head or one token for all."""
    counts = [33, 130]
    q, k, v = data(counts, counts, 4, 2, 64, dtype, 3)
    wide = torch.full((163, 10, 72), NAN, dtype=dtype, device="cuda")
    wide[:, :4, 8:], wide[:, 4:6, 8:], wide[:, 7:9, :64] = q.cuda(), k.cuda(), v.cuda()
    y = torch.full((6, 163, 64), 7.0, dtype=dtype, device="cuda")
    lse = torch.zeros(163, 4, device="cuda")
    first = starts(counts).cuda()
    ctx.attend(wide[:, :4, 8:], wide[:, 4:6, 8:], wide[:, 7:9, :64], y.transpose(0, 1)[:, 1:5], first, 0.125, lse=lse, stream=stream())
    assert_attention(y.transpose(0, 1)[:, 1:5].cpu(), lse.cpu(), right(q, k, v, counts, counts, 0.125))
    assert bool((y[0] == 7).all()) and bool((y[5] == 7).all())
    same = lambda t: t[:1].expand(t.shape)
    out = torch.zeros(163, 4, 64, dtype=dtype, device="cuda")
    ctx.attend(same(q.cuda()), k.cuda()[:, :1].expand(163, 2, 64), same(v.cuda()), out, first, 0.125, stream=stream())
    assert_attention(out.cpu(), None, right(same(q), k[:, :1].expand(163, 2, 64), same(v), counts, counts, 0.125))


def test_rows_far_apart(ctx):
    """Offsets beyond 32 bits, of elements and of bytes: queries and results 2^30 elements apart, keys and values 2^23, as far as they may be."""
    q, k, v = data([3, 0], [300, 3], 2, 1, 64, F16, 4)
    far, near = (1 << 30) + 64, 1 << 23
    store = torch.empty(max(far * 2, near * 303) + 4096, dtype=F16, device="cuda")
    views = [store.as_strided((n, h, 64), (by, 64, 1), storage_offset=at) for n, h, by, at in ((3, 2, far, 0), (303, 1, near, 512), (303, 1, near, 576), (3, 2, far, 256))]
    for to, x in zip(views, (q, k, v)):
        to.copy_(x)
    ctx.attend(*views, starts([3, 0]).cuda(), 0.125, first_k=starts([300, 3]).cuda(), stream=stream())
    assert_attention(views[3].cpu(), None, right(q, k, v, [3, 0], [300, 3], 0.125))


def test_results_of_parts_join(ctx):
    """Softmaxes over two parts of the keys, joined by their lse, are that over all."""
    n, m = 50, 300
    q, k, v = data([n], [m], 2, 2, 64, F16, 4)
    out = []
    for a, b in ((0, 170), (170, m)):
        y, lse = torch.zeros(q.shape, dtype=F16, device="cuda"), torch.zeros(n, 2, device="cuda")
        ctx.attend(q.cuda(), k[a:b].cuda(), v[a:b].cuda(), y, starts([n]).cuda(), 0.125, first_k=starts([b - a]).cuda(), causal=False, lse=lse, stream=stream())
        out.append((y.cpu().double(), lse.cpu().double()))
    total = torch.logaddexp(out[0][1], out[1][1])
    y = sum(o[0] * torch.exp(o[1] - total)[..., None] for o in out)
    ry, rl, oy, ol = right(q, k, v, [n], [m], 0.125, False)
    assert bool(((total - rl).abs() <= 2 * ol + 1e-6).all())
    assert bool(((y - ry).abs() <= 2 * (oy + HALF_STEP[F16] * 2 * (v.abs().max().double()))).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_same_bits_every_time_on_two_streams_at_once_and_replayed(ctx, dtype):
    counts, counts_k = [130, 1, 300, 64], [130, 200, 310, 64]
    q, k, v = (t.cuda() for t in data(counts, counts_k, 8, 2, 128, dtype, 4))
    first, first_k = starts(counts).cuda(), starts(counts_k).cuda()

    def go(out, s):
        ctx.attend(q, k, v, out[0], first, 0.1, first_k=first_k, lse=out[1], stream=s)
    outs = [(torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")) for _ in range(7)]
    go(outs[6], stream())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(6):
        go(outs[i], streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o[0], outs[6][0]) and torch.equal(o[1], outs[6][1]) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(outs[0], stream())
    for i in range(3):
        q.copy_(q.roll(1 + i, 0))
        first.copy_(starts([[100, 50, 300, 45], [1, 1, 1, 492], [495, 0, 0, 0]][i]).cuda())
        go(outs[1], stream())
        torch.cuda.synchronize()
        outs[0][0].zero_(), outs[0][1].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_nothing_to_do(ctx):
    z = torch.zeros(0, 2, 64, dtype=F16, device="cuda")
    ctx.attend(z, z, z, z, torch.zeros(3, dtype=torch.int32, device="cuda"), 0.1, stream=stream())
    y, q = torch.full((3, 2, 64), 7.0, dtype=F16, device="cuda"), torch.ones(3, 2, 64, dtype=F16, device="cuda")
    ctx.attend(q, z, z, y, torch.tensor([0, 2], dtype=torch.int32).cuda(), 0.1, first_k=torch.zeros(2, dtype=torch.int32, device="cuda"), stream=stream())
    assert not bool(y[:2].any()) and bool((y[2] == 7).all())
