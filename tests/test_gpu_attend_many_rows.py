"""cw_attend where the rows fill the GPU and no waves share them (more than 320 workgroups of 128 rows), against 64 bits: types, head sizes, several tiles of keys with and without
masks, histories, windows, what is not seen, scores that rise and fall, strides, far rows, streams and graphs."""
import math

import pytest
import torch

import paper_2006_02464_amd as cw
from attend_bounds import assert_close, attention
from attend_refs import BF16, F16, HALF_STEP, INF, NAN, seen_causal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = cw.Context(workspace_bytes=16 << 20, io_bytes=1 << 20, weight_pool_bytes=16 << 20, load_staging_bytes=1 << 20)
    yield c
    c.destroy()


def stream():
    return torch.cuda.current_stream()


def starts(counts):
    return torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32)


def data(counts, counts_k, heads, kv_heads, dim, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    by = 1.0 + 9.0 * (torch.rand(kv_heads, dim, generator=g) < 0.03)
    make = lambda n, h, by: (torch.randn(n, h, dim, generator=g) * by).to(dtype)
    return make(sum(counts), heads, 1.0), make(sum(counts_k), kv_heads, by), make(sum(counts_k), kv_heads, 1.0)


def right(q, k, v, counts, counts_k, scale, causal=True, window=0):
    """A weight is rounded to the values' type: half a step of it, and of fp16 2^-25 of the largest weight at most where fp16's numbers end."""
    parts, a, b = [], 0, 0
    for n, m in zip(counts, counts_k):
        if n:
            parts.append(attention(q[a:a + n], k[b:b + m], v[b:b + m], scale, seen_causal(n, m, causal, window), HALF_STEP[q.dtype], 2.0 ** -25 if q.dtype == F16 else 0.0))
        a, b = a + n, b + m
    return tuple(torch.cat([p[j] for p in parts]) for j in range(4))


def whole(q, k, counts):
    """Of each wave its rows alone: the bound that the call goes by."""
    assert q.shape[0] * q.shape[1] // 128 + len(counts) * k.shape[1] > 320


def check(ctx, q, k, v, counts, counts_k, scale=None, causal=True, window=0, what=""):
    whole(q, k, counts)
    scale = 1.0 / math.sqrt(q.shape[2]) if scale is None else scale
    y, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    same = list(counts) == list(counts_k)
    ctx.attend(q.cuda(), k.cuda(), v.cuda(), y, starts(counts).cuda(), scale, first_k=None if same else starts(counts_k).cuda(), causal=causal, window=window, lse=lse, stream=stream())
    assert_close(y.cpu(), lse.cpu(), right(q, k, v, counts, counts_k, scale, causal, window), what)


COUNTS = [300, 1, 2, 0, 31, 64, 65, 127, 128, 129, 257, 330, 33]
SIZES = [(16, 16, 64), (32, 16, 96), (24, 24, 80), (48, 16, 128), (16, 16, 192), (18, 18, 240), (32, 16, 256), (17, 17, 16)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads, kv_heads, dim", SIZES)
def test_packed_lengths_heads_and_sizes(ctx, dtype, causal, heads, kv_heads, dim):
    q, k, v = data(COUNTS, COUNTS, heads, kv_heads, dim, dtype, dim)
    check(ctx, q, k, v, COUNTS, COUNTS, causal=causal)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads, kv_heads, dim", [(32, 8, 128), (64, 4, 64), (16, 16, 256)])
def test_one_long_prompt(ctx, dtype, heads, kv_heads, dim):
    """Sixteen tiles and more, nearly all of them without masks."""
    n = 1025 if heads > 16 else 2500
    q, k, v = data([n], [n], heads, kv_heads, dim, dtype, dim)
    pad = [1] * (0 if n * heads // 128 + kv_heads > 320 else 20)
    if pad:
        q2, k2, v2 = data(pad, pad, heads, kv_heads, dim, dtype, 1)
        q, k, v = torch.cat([q, q2]), torch.cat([k, k2]), torch.cat([v, v2])
    check(ctx, q, k, v, [n] + pad, [n] + pad)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads, kv_heads, dim", [(32, 32, 64), (32, 32, 96), (64, 32, 128), (32, 32, 192), (32, 32, 256)])
def test_other_numbers_of_keys_than_of_queries(ctx, dtype, causal, heads, kv_heads, dim):
    """Parts behind their histories; fewer keys than queries, whose first rows see nothing; no keys."""
    counts, counts_k = [1, 40, 130, 3, 70, 5, 0, 64, 200], [500, 41, 300, 0, 20, 5, 10, 193, 100]
    q, k, v = data(counts, counts_k, heads, kv_heads, dim, dtype, 3)
    check(ctx, q, k, v, counts, counts_k, causal=causal)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("window", [1, 33, 64, 100, 129, 1000])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_windows(ctx, dtype, window, dim):
    counts, counts_k = [1, 40, 130, 300, 70, 0, 64], [500, 41, 300, 300, 20, 10, 193]
    q, k, v = data(counts, counts_k, 48, 48, dim, dtype, 3)
    check(ctx, q, k, v, counts, counts_k, window=window)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_what_is_not_seen_has_no_effect(ctx, dtype, value, dim):
    """Keys and values behind a query in its own tile, before its window, of the neighbours: queries that do not see them are as if they were numbers, others NaN or what the values say."""
    counts, heads = [70, 200, 40], 96
    q, k, v = data(counts, counts, heads, heads, dim, dtype, 7)
    whole(q, k, counts)
    bad_k, bad_v = torch.zeros(k.shape, dtype=torch.bool), torch.zeros(v.shape, dtype=torch.bool)
    bad_k[70 + 90:70 + 92, 1], bad_v[70 + 100, 0, 3], bad_v[70 + 130, 0, :], bad_v[70 + 131, 1, 7] = True, True, True, True
    bad_k[269, 0, 0], bad_v[269, 1], bad_k[0, 0, 0], bad_v[69, 0, 1], bad_v[5, 95] = True, True, True, True, True
    spoilt_k, spoilt_v = torch.where(bad_k, torch.tensor(value, dtype=dtype), k), torch.where(bad_v, torch.tensor(value, dtype=dtype), v)
    for window in (0, 37, 3):
        y, lse = torch.zeros(q.shape, dtype=dtype, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
        ctx.attend(q.cuda(), spoilt_k.cuda(), spoilt_v.cuda(), y, starts(counts).cuda(), 0.1, window=window, lse=lse, stream=stream())
        ref = right(q, k, v, counts, counts, 0.1, True, window)
        y, lse = y.cpu(), lse.cpu()
        a = 0
        sees_k, sees_v = torch.zeros(q.shape[:2], dtype=torch.bool), torch.zeros(q.shape, dtype=torch.bool)
        for n in counts:
            seen = seen_causal(n, n, True, window).double()
            sees_k[a:a + n] = (torch.einsum("ij,jh->ih", seen, bad_k[a:a + n].any(2).double()) > 0)
            sees_v[a:a + n] = (torch.einsum("ij,jhd->ihd", seen, bad_v[a:a + n].double()) > 0)
            a += n
        clean = ~sees_k[..., None] & ~sees_v
        fill = lambda got, want: torch.where(clean, got.double(), want)
        assert_close(fill(y, ref[0]).to(dtype), torch.where(sees_k, ref[1], lse.double()), (ref[0], ref[1], ref[2] + HALF_STEP[dtype] * ref[0].abs(), ref[3]), window)
        spoilt = sees_v & ~sees_k[..., None]
        assert bool((y[spoilt].isnan() if value != value else y[spoilt] == value).all())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("what", ["equal", "one far above", "rising", "falling", "far below zero", "huge", "negative scale", "zero scale"])
@pytest.mark.parametrize("dim", [64, 256])
def test_scores_of_all_kinds(ctx, dtype, what, dim):
    n, heads = 520, 80
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(n, heads, dim, generator=g) for _ in range(3))
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
    else:
        scale = 0.0
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    check(ctx, q, k, v, [n], [n], scale, True)
    check(ctx, q, k, v, [n], [n], scale, False)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_strides(ctx, dtype):
    """Parts of a projection's result; heads ahead of tokens."""
    counts, heads, kv_heads = [33, 130, 300], 96, 96
    q, k, v = data(counts, counts, heads, kv_heads, 64, dtype, 3)
    whole(q, k, counts)
    total = sum(counts)
    wide = torch.full((total, 3 * heads + 2, 72), NAN, dtype=dtype, device="cuda")
    wide[:, :heads, 8:], wide[:, heads:2 * heads, 8:], wide[:, 2 * heads + 1:3 * heads + 1, :64] = q.cuda(), k.cuda(), v.cuda()
    y = torch.full((heads + 2, total, 64), 7.0, dtype=dtype, device="cuda")
    lse = torch.zeros(total, heads, device="cuda")
    ctx.attend(wide[:, :heads, 8:], wide[:, heads:2 * heads, 8:], wide[:, 2 * heads + 1:3 * heads + 1, :64], y.transpose(0, 1)[:, 1:heads + 1], starts(counts).cuda(), 0.125, lse=lse, stream=stream())
    assert_close(y.transpose(0, 1)[:, 1:heads + 1].cpu(), lse.cpu(), right(q, k, v, counts, counts, 0.125))
    assert bool((y[0] == 7).all()) and bool((y[heads + 1] == 7).all())


def test_rows_far_apart(ctx):
    """Keys and values 2^23 elements apart, queries and results 2^27."""
    counts, counts_k, heads = [3, 0, 7], [150, 3, 60], 112
    q, k, v = data(counts, counts_k, heads, heads, 64, F16, 4)
    whole(q, k, counts)
    far, near = 1 << 27, 1 << 23
    store = torch.empty(max(far * 10, near * 213) + (1 << 16), dtype=F16, device="cuda")
    part = heads * 64
    views = [store.as_strided((n, heads, 64), (by, 64, 1), storage_offset=at) for n, by, at in ((10, far, 0), (213, near, part), (213, near, 2 * part), (10, far, 3 * part))]
    for to, x in zip(views, (q, k, v)):
        to.copy_(x)
    ctx.attend(*views, starts(counts).cuda(), 0.125, first_k=starts(counts_k).cuda(), stream=stream())
    assert_close(views[3].cpu(), None, right(q, k, v, counts, counts_k, 0.125))


@pytest.mark.parametrize("dtype, dim", [(F16, 128), (BF16, 128), (BF16, 256)])
def test_same_bits_every_time_on_two_streams_at_once_and_replayed(ctx, dtype, dim):
    counts, counts_k = [130, 1, 300, 64], [130, 200, 310, 64]
    q, k, v = (t.cuda() for t in data(counts, counts_k, 96, 96, dim, dtype, 4))
    whole(q, k, counts)
    first, first_k = starts(counts).cuda(), starts(counts_k).cuda()

    def go(out, s):
        ctx.attend(q, k, v, out[0], first, 0.1, first_k=first_k, lse=out[1], stream=s)
    outs = [(torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")) for _ in range(5)]
    go(outs[4], stream())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(4):
        go(outs[i], streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o[0], outs[4][0]) and torch.equal(o[1], outs[4][1]) for o in outs)
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
