"""cw_attend_one and cw_attend at the ends of the numbers: values that are none beside weights of 0, exponents from end to end, scales next to 0."""
import math

import pytest
import torch

import paper_2006_02464_amd as cw
from attend_bounds import assert_close, attention
from attend_refs import BF16, E4M3, F16, F32, HALF_STEP, INF, NAN, Pages, seen_causal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = cw.Context(workspace_bytes=16 << 20, io_bytes=1 << 20, weight_pool_bytes=16 << 20, load_staging_bytes=1 << 20)
    yield c
    c.destroy()


@pytest.fixture(scope="module")
def space(ctx):
    return torch.zeros(ctx.attend_one_workspace_bytes(), dtype=torch.uint8, device="cuda")


def stream():
    return torch.cuda.current_stream()


def one(ctx, pool, q, scale, workspace):
    handle, gpu = pool.cuda(ctx)
    y, lse = torch.zeros(q.shape, dtype=q.dtype, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
    ctx.attend_one(q.cuda(), handle, pool.table.cuda(), torch.tensor(pool.lengths, dtype=torch.int32).cuda(), y, scale, lse=lse, workspace=workspace, stream=stream())
    return y.cpu(), lse.cpu()


@pytest.mark.parametrize("kept", [F16, BF16, E4M3])
@pytest.mark.parametrize("value", [NAN, INF])
@pytest.mark.parametrize("lengths", [[3000], [3000, 2500], [3000] + [40] * 70])
def test_values_that_are_none_beside_weights_of_0(ctx, space, kept, value, lengths):
    """A seen value that is no number makes its number of the result NaN however far its weight is below the largest (2^-200 here), whether parts of the sequence meet or one workgroup has it all."""
    x = F16 if kept == E4M3 else kept
    pool = Pages(lengths, 2, 16, 64, kept, seed=2).fill(5, loud=False)
    page, at = int(pool.table[0, 2990 // 16]), 2990 % 16
    k = torch.zeros(1, 2, 64, dtype=x)
    k[..., 0] = 200.0
    rest = Pages([1], 2, 16, 64, kept, spare=0)
    rest.write(0, k, k, 1)
    pool.k[page, :, at] = rest.k[0, :, 0]
    if kept == E4M3:
        pool.k_exp[page, :, at] = rest.k_exp[0, :, 0]
    pool.v[int(pool.table[0, 0]), 1, 5, 7] = value if kept != E4M3 else 0x7f
    q = torch.zeros(len(lengths), 4, 64, dtype=x)
    q[..., 0] = 1.0
    for workspace in (space, None):
        y, lse = one(ctx, pool, q, 1.0, workspace)
        want = torch.zeros(y.shape, dtype=torch.bool)
        want[0, 2:, 7] = True
        assert torch.equal(y.isnan(), want), workspace is not None
        assert bool(y[~want].isfinite().all()) and bool(lse.isfinite().all())


@pytest.mark.parametrize("x", [F16, BF16])
@pytest.mark.parametrize("e_k, e_v", [(127, 0), (127, 3), (120, 60), (127, 127), (127, 200), (110, 230), (0, 127), (140, 225)])
@pytest.mark.parametrize("lengths", [[40, 1, 3], [2500, 300]])
def test_exponents_from_end_to_end(ctx, space, x, e_k, e_v, lengths):
    """Codes times 2^-127 up to 2^103, of keys as far as their scores are numbers.  Results of fp16 end in 0 or infinity, those of bf16 are ordinary numbers, or its smallest."""
    pool = Pages(lengths, 2, 16, 64, E4M3, seed=2).fill(5, loud=False)
    pool.k_exp[pool.k_exp < 255] = e_k
    pool.v_exp[pool.v_exp < 255] = e_v
    q = (torch.randn(len(lengths), 4, 64, generator=torch.Generator().manual_seed(3))).to(x)
    scale = 2.0 ** -8 * 2.0 ** min(100, max(-20, 127 - e_k))      # codes are up to 448
    refs = []
    for i, n in enumerate(lengths):
        k, v, _ = pool.read(i, 0, n)
        refs.append(attention(q[i:i + 1], k, v, scale, torch.ones(1, n, dtype=torch.bool), 2.0 ** -11, 2.0 ** -36))
    ry, rl, off_y, off_l = (torch.cat([r[j] for r in refs]) for j in range(4))
    for workspace in (space, None):
        y, lse = one(ctx, pool, q, scale, workspace)
        ends = ry.abs() >= torch.finfo(x).max
        assert bool((y.isinf() | (y.abs() == torch.finfo(x).max))[ends].all())
        off = off_y + 2.0 ** -149 * 2                        # fp32's own end, of the result and of a sum
        assert_close(torch.where(ends, torch.zeros_like(y), y), lse, (torch.where(ends, 0.0, ry), rl, off, off_l), workspace is not None)


def far_scores(n, heads, kv_heads, dim, scale):
    """Queries and keys of bf16 whose product is up to 10^38, which `scale` brings back."""
    g = torch.Generator().manual_seed(6)
    q, k, v = torch.randn(n, heads, dim, generator=g), torch.randn(n, kv_heads, dim, generator=g), torch.randn(n, kv_heads, dim, generator=g)
    q, k = q * 1e-3, k * 1e-3
    q[..., 0], k[..., 0] = 1e19, 1e19 * (2.0 * torch.rand(n, kv_heads, generator=g) - 1.0)
    return q.to(BF16), k.to(BF16), v.to(BF16)


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45, 1e-40, -1e-39, 1e-38, -5e-38, 2e-37])
def test_scales_next_to_0(ctx, space, scale):
    """Down to fp32's last numbers the scale counts as it is, and 0 as 0: softmaxes over equal scores."""
    as_given = float(torch.tensor(scale, dtype=torch.float32))
    for heads, kv_heads in ((2, 1), (84, 84)):               # waves that share rows, and do not
        n = 500
        q, k, v = far_scores(n, heads, kv_heads, 64, scale)
        for causal in (True, False):
            y, lse = torch.zeros(q.shape, dtype=BF16, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
            ctx.attend(q.cuda(), k.cuda(), v.cuda(), y, torch.tensor([0, n], dtype=torch.int32).cuda(), scale, causal=causal, lse=lse, stream=stream())
            assert_close(y.cpu(), lse.cpu(), attention(q, k, v, as_given, seen_causal(n, n, causal), HALF_STEP[BF16], 0.0), (heads, causal))
    for kept in (BF16, E4M3):
        lengths = [400, 1000]
        pool, refs = Pages(lengths, 2, 16, 64, kept, seed=2), []
        for i, n in enumerate(lengths):
            q, k, v = far_scores(n, 4, 2, 64, scale)
            pool.write(i, k, v, n)
            k, v, _ = pool.read(i, 0, n)
            refs.append(attention(q[:1], k, v, as_given, torch.ones(1, n, dtype=torch.bool), 2.0 ** -11, 2.0 ** -35))
        y, lse = one(ctx, pool, torch.stack([q[0], q[0]]), scale, space)
        assert_close(y, lse, tuple(torch.cat([r[j] for r in refs]) for j in range(4)), kept)


@pytest.mark.parametrize("sequences", [252, 254, 255])
def test_the_workspace_that_serves_every_call(ctx, sequences):
    """More than attend_one_workspace_bytes() changes nothing: not a bit of the results, and what lies behind them stays."""
    lengths = [i * 13 % 50 for i in range(sequences)]
    lengths[0], lengths[100], lengths[sequences - 1] = 4096, 4000, 4096
    pool = Pages(lengths, 8, 64, 128, E4M3, seed=2).fill(5)
    handle, gpu = pool.cuda(ctx)
    table, lens = pool.table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
    q = torch.randn(sequences, 128, 128, generator=torch.Generator().manual_seed(3)).half().cuda()
    most, out = ctx.attend_one_workspace_bytes(), []
    for size in (most, 3 * most):
        space = torch.full((size,), 0x5a, dtype=torch.uint8, device="cuda")
        space[:cw.CW_ATTEND_COUNTERS] = 0
        y, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
        ctx.attend_one(q, handle, table, lens, y, 0.08, lse=lse, workspace=space, stream=stream())
        assert bool((space[most:] == 0x5a).all())
        out.append((y, lse))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


@pytest.mark.parametrize("kept", [F16, E4M3])
def test_pools_of_no_pages(ctx, space, kept):
    """Nothing is written, zeros are read, rows see nothing."""
    k = torch.zeros(0, 2, 16, 64, dtype=kept, device="cuda")
    exps = [torch.zeros(0, 2, 16, dtype=torch.uint8, device="cuda") if kept == E4M3 else None for _ in range(2)]
    cache = ctx.cache(k, k.clone(), *exps)
    table, lens = torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.tensor([0, 5, 20], dtype=torch.int32).cuda()
    x = torch.ones(3, 2, 64, dtype=F16, device="cuda")
    z = x.clone()
    ctx.cache_write(x, z, cache, table, lens, stream=stream())
    ctx.cache_read(cache, table, lens, x, z, stream=stream())
    assert not bool(x.any()) and not bool(z.any())
    q, y = (torch.ones(3, 4, 64, dtype=F16, device="cuda") for _ in range(2))
    lse = torch.ones(3, 4, device="cuda")
    ctx.attend_one(q, cache, table, lens, y, 0.1, lse=lse, workspace=space, stream=stream())
    assert not bool(y.any()) and bool((lse == -INF).all())
