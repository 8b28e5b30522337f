"""cw_cache_write and cw_cache_read against the definition, bit for bit: types, head sizes, pages, tables with holes, rows that are none, layouts, far pages, graphs."""
import math

import pytest
import torch

import paper_2006_02464_amd as cw
from attend_refs import BF16, E4M3, F16, F32, INF, NAN, Pages, coded, decoded

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


def same_bits(a, b):
    a, b = a.cpu(), b.cpu()
    if a.dtype == torch.uint8 or b.dtype == torch.uint8 or a.dtype == E4M3:
        a, b = a.view(torch.uint8), b.view(torch.uint8)
        nan = (a & 0x7f == 0x7f) & (b & 0x7f == 0x7f)
        return bool(((a == b) | nan).all())
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def rows(counts, heads, dim, dtype, seed, big=1.0):
    g = torch.Generator().manual_seed(seed)
    make = lambda: (torch.randn(sum(counts), heads, dim, generator=g) * big * 2.0 ** torch.randint(-6, 7, (sum(counts), heads, 1), generator=g)).to(dtype)
    return make(), make()


def check(ctx, pool, lengths, counts, k, v, first, layout="head first", exps=True):
    """Writes, and reads back what was written."""
    handle, gpu = pool.cuda(ctx, layout)
    table, lens = pool.table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
    kd, vd, fd = k.cuda(), v.cuda(), None if first is None else first.cuda()
    ctx.cache_write(kd, vd, handle, table, lens, first=fd, stream=stream())
    offset = 0 if first is None else int(first[0])
    at = offset
    for i, n in enumerate(counts):
        pool.write(i, k[at:at + n], v[at:at + n], lengths[i])
        at += n
    for got, want in zip(gpu, (pool.k, pool.v, pool.k_exp, pool.v_exp)):
        assert (got is None) == (want is None)
        if got is not None:
            assert same_bits(got, want)
    back_k, back_v = torch.full_like(kd, 7.0), torch.full_like(vd, 7.0)
    ctx.cache_read(handle, table, lens, back_k, back_v, first=fd, stream=stream())
    want_k, want_v = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    at = offset
    for i, n in enumerate(counts):
        rk, rv, _ = pool.read(i, lengths[i] - n, lengths[i])
        want_k[at:at + n], want_v[at:at + n] = rk.to(k.dtype), rv.to(v.dtype)
        at += n
    assert same_bits(back_k, want_k) and same_bits(back_v, want_v)


@pytest.mark.parametrize("x, kept", [(F16, F16), (BF16, BF16), (F32, BF16), (F32, F16), (F16, E4M3), (BF16, E4M3), (F32, E4M3), (BF16, F16)])
@pytest.mark.parametrize("heads, dim, page", [(1, 16, 1), (3, 64, 16), (8, 128, 16), (5, 80, 8), (2, 256, 64), (7, 48, 4), (1, 240, 2), (16, 96, 128)])
def test_types_and_sizes(ctx, x, kept, heads, dim, page):
    lengths, counts = [5, 33, 1, 64, 17], [5, 12, 1, 64, 3]
    pool = Pages(lengths, heads, page, dim, kept, seed=dim)
    k, v = rows(counts, heads, dim, x, dim + page)
    check(ctx, pool, lengths, counts, k, v, starts(counts))


@pytest.mark.parametrize("kept", [F16, E4M3])
@pytest.mark.parametrize("sequences", [1, 2, 63, 64, 65, 200, 4097])
def test_one_token_each_and_many_sequences(ctx, kept, sequences):
    lengths = [1 + i * 7 % 23 for i in range(sequences)]
    k, v = rows([1] * sequences, 2, 32, F16, sequences)
    check(ctx, Pages(lengths, 2, 8, 32, kept, seed=3), lengths, [1] * sequences, k, v, None)
    counts = [i % 3 if i % 3 <= lengths[i] else 0 for i in range(sequences)]      # some have none
    k, v = rows(counts, 2, 32, F16, sequences + 1)
    check(ctx, Pages(lengths, 2, 8, 32, kept, seed=4), lengths, counts, k, v, starts(counts))


@pytest.mark.parametrize("kept", [BF16, E4M3])
def test_holes_and_rows_that_are_none(ctx, kept):
    """Pages that are not there or not numbers of pages, tokens behind the table's end and before the sequence's beginning, rows before the first sequence and behind the last."""
    lengths, counts = [40, 3, 0, 30, 9], [40, 8, 4, 30, 2]
    pool = Pages([40, 3, 0, 30, 9], 2, 8, 64, kept, seed=1, table_pages=4)      # the first sequence has five pages' tokens
    pool.table[0, 1] = -1
    pool.table[3, 0], pool.table[3, 2], pool.table[3, 3] = pool.pages, 2 ** 31 - 1, -2 ** 31
    k, v = rows([6] + counts + [5], 2, 64, BF16, 8)
    first = starts(counts) + 6
    check(ctx, pool, lengths, counts, k, v, first)


def test_lengths_that_are_no_lengths(ctx):
    for n in (-1, -2 ** 31, 2 ** 31 - 1):
        pool = Pages([8, 8], 1, 8, 32, F16)
        k, v = rows([3, 3], 1, 32, F16, 2)
        check(ctx, pool, [n, 8], [3, 3], k, v, starts([3, 3]))


@pytest.mark.parametrize("x", [F16, BF16, F32])
def test_numbers_at_the_ends(ctx, x):
    """Zeros, subnormals, the largest, NaN and infinities, magnitudes just at and above 448 times a power of two, ties of the rounding."""
    info = torch.finfo(x)
    dim = 32
    z = torch.zeros(14, 1, dim)
    z[1, 0, 3] = info.max
    z[2, 0, 3], z[2, 0, 4] = info.smallest_normal, info.smallest_normal / 4
    z[3, 0, :] = info.smallest_normal * info.eps
    z[4, 0, 1], z[4, 0, 2] = NAN, 5.0
    z[5, 0, 1], z[5, 0, 2], z[5, 0, 3] = INF, -INF, 3.0
    z[6, 0, :] = NAN
    z[7, 0, 0], z[7, 0, 1:] = 448.0, torch.linspace(0, 2, 31)
    z[8, 0, 0], z[8, 0, 1:] = 450.0, torch.linspace(-2, 2, 31)
    z[9, 0, 0], z[9, 0, 1:17] = 448.0, 16.0 + torch.arange(16.0)                  # ties: steps of 2 there
    z[10, 0, 0], z[10, 0, 1:17] = 448.0, (torch.arange(16.0) + 0.5) * 2.0 ** -9     # ties among the smallest codes
    z[11, 0, 0], z[11, 0, 1] = 1.75 * 2.0 ** -3, -1.75 * 2.0 ** -3
    z[12, 0, 0] = -0.0
    z[13, 0, :] = torch.linspace(-448, 448, 32)
    z = z.to(x)
    for kept in (E4M3,) if x != BF16 else (E4M3, BF16):
        pool = Pages([14], 1, 4, dim, kept)
        check(ctx, pool, [14], [14], z, z.flip(0), starts([14]))


def test_the_definition_of_the_codes():
    """coded(), which the others are held to, against torch's own rounding to e4m3."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(500, 64, generator=g) * 2.0 ** torch.randint(-20, 20, (500, 1), generator=g)
    codes, exps = coded(x)
    assert torch.equal(codes.view(E4M3).float(), (x.double() * torch.exp2(127.0 - exps.double())[:, None]).float().to(E4M3).float())
    assert bool((codes.view(E4M3).float().abs().amax(1) > 223).all())
    assert bool(((decoded(codes, exps) - x).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -10 * torch.exp2(exps.double() - 127)[:, None]).all())


@pytest.mark.parametrize("kept", [F16, E4M3])
def test_layouts_and_strides(ctx, kept):
    lengths, counts = [20, 9], [20, 9]
    k, v = rows(counts, 4, 64, F16, 5)
    check(ctx, Pages(lengths, 4, 16, 64, kept), lengths, counts, k, v, starts(counts), layout="token first")
    # rows that are parts of a projection's result; keys and values of a page side by side
    pool = Pages(lengths, 4, 16, 64, kept)
    both = torch.zeros(pool.pages, 2, 4, 16, 64, dtype=torch.uint8 if kept == E4M3 else kept, device="cuda")
    both[:, 0], both[:, 1] = pool.k.cuda(), pool.v.cuda()
    both = both.view(kept)
    exps = [e.cuda() if e is not None else None for e in (pool.k_exp, pool.v_exp)]
    handle = ctx.cache(both[:, 0], both[:, 1], k_exp=exps[0], v_exp=exps[1])
    wide = torch.full((29, 16, 64), NAN, dtype=F16, device="cuda")
    wide[:, 8:12], wide[:, 12:16] = k.cuda(), v.cuda()
    lens, table, first = torch.tensor(lengths, dtype=torch.int32).cuda(), pool.table.cuda(), starts(counts).cuda()
    ctx.cache_write(wide[:, 8:12], wide[:, 12:16], handle, table, lens, first=first, stream=stream())
    for i in range(2):
        a = int(first[i])
        pool.write(i, k[a:a + counts[i]], v[a:a + counts[i]], lengths[i])
    assert same_bits(both[:, 0].contiguous(), pool.k) and same_bits(both[:, 1].contiguous(), pool.v)
    back = torch.full((29, 16, 64), 7.0, dtype=F32, device="cuda")
    ctx.cache_read(handle, table, lens, back[:, 2:6], back[:, 7:11], first=first, stream=stream())
    want_k, want_v = (torch.cat([pool.read(i, 0, lengths[i])[j] for i in range(2)]).float().cuda() for j in (0, 1))
    assert torch.equal(back[:, 2:6], want_k) and torch.equal(back[:, 7:11], want_v)
    assert bool((back[:, :2] == 7).all()) and bool((back[:, 6] == 7).all()) and bool((back[:, 11:] == 7).all())


@pytest.mark.parametrize("kept", [F16, E4M3])
def test_pages_far_apart(ctx, kept):
    """Offsets beyond 32 bits."""
    far = (1 << 31) + 4096
    pool = Pages([20, 7], 2, 8, 32, kept, spare=0)
    size = 1 if kept == E4M3 else 2
    store = torch.empty((far * (pool.pages - 1) + (1 << 16)) * size, dtype=torch.uint8, device="cuda").view(kept)
    shape, strides = (pool.pages, 2, 8, 32), (far, 256, 32, 1)
    k, v = store.as_strided(shape, strides), store.as_strided(shape, strides, storage_offset=1024)
    k.view(torch.uint8).copy_(pool.k.view(torch.uint8)) if size == 1 else k.copy_(pool.k)
    v.view(torch.uint8).copy_(pool.v.view(torch.uint8)) if size == 1 else v.copy_(pool.v)
    exps = [e.cuda() if e is not None else None for e in (pool.k_exp, pool.v_exp)]
    handle = ctx.cache(k, v, k_exp=exps[0], v_exp=exps[1])
    x, z = rows([20, 7], 2, 32, F16, 4)
    lens, first = torch.tensor([20, 7], dtype=torch.int32).cuda(), starts([20, 7])
    ctx.cache_write(x.cuda(), z.cuda(), handle, pool.table.cuda(), lens, first=first.cuda(), stream=stream())
    pool.write(0, x[:20], z[:20], 20)
    pool.write(1, x[20:], z[20:], 7)
    back_k, back_v = torch.zeros(27, 2, 32, device="cuda"), torch.zeros(27, 2, 32, device="cuda")
    ctx.cache_read(handle, pool.table.cuda(), lens, back_k, back_v, first=first.cuda(), stream=stream())
    want = [torch.cat([pool.read(0, 0, 20)[j], pool.read(1, 0, 7)[j]]).float() for j in (0, 1)]
    assert torch.equal(back_k.cpu(), want[0]) and torch.equal(back_v.cpu(), want[1])


@pytest.mark.parametrize("kept", [BF16, E4M3])
def test_captured_and_on_another_stream(ctx, kept):
    lengths = [9, 30, 1]
    pool = Pages([48, 48, 48], 2, 8, 64, kept)
    handle, gpu = pool.cuda(ctx)
    lens, table = torch.tensor(lengths, dtype=torch.int32).cuda(), pool.table.cuda()
    k, v = (t.cuda() for t in rows([1, 1, 1], 2, 64, BF16, 1))
    out = [torch.zeros(3, 2, 64, dtype=BF16, device="cuda") for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ctx.cache_write(k, v, handle, table, lens, stream=stream())
        ctx.cache_read(handle, table, lens, out[0], out[1], stream=stream())
    other = torch.cuda.Stream()
    for step in range(4):
        nk, nv = rows([1, 1, 1], 2, 64, BF16, step + 9)
        k.copy_(nk), v.copy_(nv)
        if step % 2:
            other.wait_stream(torch.cuda.current_stream())
            ctx.cache_write(k, v, handle, table, lens, stream=other)
            ctx.cache_read(handle, table, lens, out[0], out[1], stream=other)
            other.synchronize()
        else:
            graph.replay()
            torch.cuda.synchronize()
        for i in range(3):
            pool.write(i, nk[i:i + 1], nv[i:i + 1], lengths[i])
            rk, rv, _ = pool.read(i, lengths[i] - 1, lengths[i])
            assert same_bits(out[0][i:i + 1], rk.to(BF16)) and same_bits(out[1][i:i + 1], rv.to(BF16))
            lengths[i] += 1
        assert same_bits(gpu[0], pool.k) and same_bits(gpu[1], pool.v)
        lens += 1


def test_nothing_to_do(ctx):
    pool = Pages([4], 2, 8, 32, F16)
    handle, gpu = pool.cuda(ctx)
    empty = torch.zeros(0, 2, 32, dtype=F16, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    ctx.cache_write(empty, empty, handle, torch.zeros(0, 3, dtype=torch.int32, device="cuda"), none, stream=stream())
    ctx.cache_write(empty, empty, handle, pool.table.cuda(), torch.tensor([4], dtype=torch.int32).cuda(), first=torch.zeros(2, dtype=torch.int32, device="cuda"), stream=stream())
    x = torch.ones(3, 2, 32, dtype=F16, device="cuda")
    ctx.cache_write(x, x, handle, torch.zeros(1, 0, dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32).cuda(), first=torch.tensor([0, 3], dtype=torch.int32).cuda(), stream=stream())
    assert same_bits(gpu[0], pool.k)
    ctx.cache_read(handle, torch.zeros(1, 0, dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32).cuda(), x, x.clone(), first=torch.tensor([0, 3], dtype=torch.int32).cuda(), stream=stream())
    assert not bool(x.any())
