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
    for at in (0, n // 2, n - few):
        q, k, v = sink(n, heads, kv_heads, dim, dtype, depth, at, few)
        first, first_k = (torch.tensor([0, x], dtype=torch.int32).cuda() for x in (few, n))
        y, lse = torch.zeros(q.shape, dtype=dtype, device="cuda"), torch.zeros(q.shape[:2], device="cuda")
        ctx.attend(q.cuda(), k.cuda(), v.cuda(), y, first, math.log(2), first_k=first_k, lse=lse, stream=stream())
        assert_close(y.cpu(), lse.cpu(), attention(q, k, v, math.log(2), seen_causal(few, n), HALF_STEP[dtype], 2.0 ** -36 if dtype == F16 else 0.0), (depth, at))
