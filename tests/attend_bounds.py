"""Attention in 64 bits, all heads at once, with bounds that have no slack for weights that a kernel leaves out."""
import math

import torch

from attend_refs import F16, HALF_STEP, INF, SMALLEST


def attention(q, k, v, scale, seen, step, least):
    """softmax(scale q k^T where seen) v of [queries][heads][dim] over [keys][kv_heads][dim], finite numbers: y, lse and the bounds of what a kernel gives before y's own rounding.

    A weight goes into the second product with `step` of itself lost and, beside that, `least` of the row's largest.  Scores are fp32 sums of dim products, (2 sqrt(dim) + 8) 2^-24 of
    A = |scale| sum |q k| (roundings that add up like chance does, but for rare luck), scaled, subtracted and raised: 2^-22 (2 A + 4).  y is a quotient of two sums of such weights: twice that;
    sums of n add (2 sqrt(n) + 8) 2^-24 each."""
    n, heads, dim = q.shape
    m, kv_heads = k.shape[:2]
    if m == 0:
        return torch.zeros(n, heads, dim, dtype=torch.float64), torch.full((n, heads), -INF, dtype=torch.float64), torch.zeros(n, heads, dim, dtype=torch.float64), torch.zeros(n, heads, dtype=torch.float64)
    spread = lambda x: x.double().transpose(0, 1).repeat_interleave(heads // kv_heads, 0)       # [heads][keys][dim]
    qh, kh, vh = q.double().transpose(0, 1), spread(k), spread(v)
    s = torch.where(seen, scale * (qh @ kh.transpose(1, 2)), -INF)
    a = torch.where(seen, abs(scale) * (qh.abs() @ kh.abs().transpose(1, 2)), 0.0).amax(2)
    top = s.amax(2)
    some = top > -INF
    e = torch.exp(s - torch.where(some, top, 0.0)[..., None])
    total = torch.where(some, e.sum(2), 1.0)
    y = (e @ vh) / total[..., None]
    lse = torch.where(some, top + torch.log(total), -INF)
    far = (2 * math.sqrt(dim) + 8) * 2.0 ** -24 * a + 2.0 ** -22 * (2 * a + 4)
    sums = (2 * math.sqrt(m) + 8) * 2.0 ** -24
    size = (e @ vh.abs()) / total[..., None]
    few = least * (seen.double() @ vh.abs()) / total[..., None]
    off_y = (2 * far + 2 * sums + step)[..., None] * size + few
    off_lse = far + sums + 2.0 ** -22 * (1 + lse.nan_to_num(0.0, 0.0, 0.0).abs())
    return tuple(t.transpose(0, 1) for t in (y, lse, off_y, off_lse))


def worst(got, want, off, dtype):
    """The largest error of numbers that are rounded to `dtype` at the end, in units of what is allowed."""
    bound = off * 1.001 + HALF_STEP[dtype] * (want.abs() + off) + SMALLEST[dtype]
    return float(((got.double() - want).abs() / bound).max()) if got.numel() else 0.0


def assert_close(y, lse, ref, what=""):
    ry, rl, off_y, off_l = ref
    far = worst(y, ry, off_y, y.dtype)
    assert far <= 1, (what, "y", far)           # NaN is not <= 1 either
    if lse is None:
        return
    assert torch.equal(lse == -INF, rl == -INF), (what, "empty rows")
    fine = rl > -INF
    far = float(((lse.double() - rl).abs() / off_l)[fine].max()) if bool(fine.any()) else 0.0
    assert far <= 1, (what, "lse", far)
