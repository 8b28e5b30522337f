"""Weights far below the largest: one key that nearly all of the softmax goes to, whose value is 0 but for one number, over many that share what is left.  The other numbers of the result are
sums of weights down to 2^-34 of the largest, which are ordinary numbers of the result's type."""
import math

import pytest
import torch

import paper_2006_02464_amd as cw
from attend_bounds import assert_close, attention
from attend_refs import BF16, E4M3, F16, HALF_STEP, INF, Pages, seen_causal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = cw.Context(workspace_bytes=16 << 20, io_bytes=1 << 20, weight_pool_bytes=16 << 20, load_staging_bytes=1 << 20)
    yield c
    c.destroy()


def stream():
    return torch.cuda.current_stream()


DEPTHS = [12, 16, 20, 26, 30, 34]      # log2 of the large weight over the others


def sink(n, heads, kv_heads, dim, dtype, depth, at, queries):
    """Scores, in units of ln 2, of `depth` at key `at` and about 0 elsewhere; scale ln 2.  Values from 512 to 1024, but 0 at the sink, whose first number is 900."""
    g = torch.Generator().manual_seed(depth + at)
    q, k = torch.randn(queries, heads, dim, generator=g) * 0.05, torch.randn(n, kv_heads, dim, generator=g) * 0.05
    q[..., 0], k[..., 0] = 1.0, 0.0
    k[at, :, 0] = depth
    v = 512.0 * (1.0 + torch.rand(n, kv_heads, dim, generator=g))
    v[at] = 0.0
    v[at, :, 0] = 900.0
    return q.to(dtype), k.to(dtype), v.to(dtype)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("depth", DEPTHS)
@pytest.mark.parametrize("heads, kv_heads, dim, n", [(4, 2, 64, 2000), (96, 48, 64, 700), (40, 40, 128, 1025)])
def test_prompts(ctx, dtype, depth, heads, kv_heads, dim, n):
    """A weight is rounded to the values' type: half a step, 2^-36 of the largest where fp16 ends (least)."""
    few = 64 if heads < 40 else n
    for at in sorted({0, n // 2, n - few}):
        q, k, v = sink(n, heads, kv_heads, dim, dtype, depth, at, few)
        first, first_k = (torch.tensor([0, x], dtype=torch.int32).cuda() for x in (few, n))
        y, lse = torch.zeros(q.shape, dtype=dtype, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
        ctx.attend(q.cuda(), k.cuda(), v.cuda(), y, first, math.log(2), first_k=first_k, lse=lse, stream=stream())
        assert_close(y.cpu(), lse.cpu(), attention(q, k, v, math.log(2), seen_causal(few, n), HALF_STEP[dtype], 2.0 ** -36 if dtype == F16 else 0.0), (depth, at))


@pytest.mark.parametrize("x, kept", [(F16, F16), (BF16, BF16), (F16, E4M3), (BF16, E4M3)])
@pytest.mark.parametrize("depth", DEPTHS)
@pytest.mark.parametrize("heads, kv_heads, dim, lengths", [(4, 2, 64, [3000, 700]), (16, 2, 128, [5000] + [150] * 70), (34, 2, 96, [100, 300])])
def test_single_tokens(ctx, x, kept, depth, heads, kv_heads, dim, lengths):
    """Of fp16 and of codes a weight has 11 bits, half a step 2^-11, and where fp16 ends half a step of 2^-25 beside a largest of 2^11 or more: 2^-36; with codes of the largest weight times its value's power
    of two, and those differ by 2 here at most, which may be either way: 2^-34.  Of bf16 it has two parts, the second at most 2^-7 of the first and off by 2^-8 of itself."""
    sequences, space = len(lengths), torch.zeros(ctx.attend_one_workspace_bytes(), dtype=torch.uint8, device="cuda")
    for place in (0.0, 0.5, 1.0) if sequences < 64 else (0.5,):
        pool, refs = Pages(lengths, kv_heads, 16, dim, kept, seed=depth), []
        q = torch.zeros(sequences, heads, dim, dtype=x)
        for i, n in enumerate(lengths):
            qi, k, v = sink(n, heads, kv_heads, dim, x, depth, min(n - 1, int(place * n)), 1)
            q[i] = qi[0]
            pool.write(i, k, v, n)
            k, v, _ = pool.read(i, 0, n)
            step, least = (2.0 ** -15, 0.0) if kept == BF16 else (2.0 ** -11, 2.0 ** -34 if kept == E4M3 else 2.0 ** -36)
            refs.append(attention(qi, k, v, math.log(2), torch.ones(1, n, dtype=torch.bool), step, least))
        ref = tuple(torch.cat([r[j] for r in refs]) for j in range(4))
        handle, gpu = pool.cuda(ctx)
        for workspace in (space, None):
            y, lse = torch.zeros(q.shape, dtype=x, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
            ctx.attend_one(q.cuda(), handle, pool.table.cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), y, math.log(2), lse=lse, workspace=workspace, stream=stream())
            assert_close(y.cpu(), lse.cpu(), ref, (depth, place, workspace is not None))
