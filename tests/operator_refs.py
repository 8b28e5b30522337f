"""Plain 64-bit forms of the single operators and the bounds that their tests use."""
import math

import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
SMALLEST = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}   # half of the smallest step


def fc4_data(rows, cin, cout, group, x_dtype, scale_dtype, zeros=False, seed=0, spread=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cin, generator=g)
    if spread:   # magnitudes over nine decades
        x = x * 10.0 ** (torch.rand(rows, cin, generator=g) * 9 - 7)
    nib = torch.randint(0, 16, (cout, cin + cin % 2), generator=g, dtype=torch.uint8)   # with an odd cin the last high nibble is anything
    groups = -(-cin // group)
    return {"x": x.to(x_dtype), "q": nib[:, 0::2] | (nib[:, 1::2] << 4), "nib": nib[:, :cin],
            "scales": ((torch.rand(cout, groups, generator=g) + 0.2) / math.sqrt(cin)).to(scale_dtype),
            "zeros": torch.randint(0, 16, (cout, groups), generator=g, dtype=torch.uint8) if zeros else None,
            "bias": torch.randn(cout, generator=g), "group": group}


def fc4_weights(d):
    cin = d["x"].shape[1]
    at = torch.arange(cin) // d["group"]
    z = d["zeros"][:, at].double() if d["zeros"] is not None else 8.0
    return (d["nib"].double() - z) * d["scales"].double()[:, at]


def fc4_ref(d):
    """y and the bound on a result before its own rounding.  Products are exact to 2^-24 each, partial sums are at most A = sum |x w| + |bias|: with
    fp32 sums in any order the roundings add up to 2 sqrt(cin) + 8 of 2^-24 A but for rare luck (their worst, all one way, is cin of them).
    fp32 activations are held in two parts, 22 bits, and bf16 and fp32 ones below 2^-36 of the row's largest may be lost."""
    x, w = d["x"].double(), fc4_weights(d)
    y = x @ w.t() + d["bias"].double()
    a = x.abs() @ w.abs().t() + d["bias"].double().abs()
    far = (2 * math.sqrt(x.shape[1]) + 8) * 2.0 ** -24 * a
    if d["x"].dtype == torch.float32:
        far = far + 2.0 ** -22 * a
    if d["x"].dtype != torch.float16:
        far = far + 2.0 ** -36 * x.abs().amax(1, keepdim=True) * w.abs().sum(1)
    return y, far


def assert_fc4(got, y, far):
    t = got.dtype
    limit = far + HALF_STEP[t] * (y.abs() + far) + SMALLEST[t]
    off = (got.double() - y).abs()
    assert bool((off <= limit).all()), "%d of %d off, worst %.3g of its bound" % (int((~(off <= limit)).sum()), off.numel(), float((off / limit).max()))


def answer_ref(x, given, top, scale):
    """The definitions of cw_answer, row by row, and the bounds on logp and entropy: with e = exp(d) off by |d| 2^-23 + 2^-22 (product and
    exponential in fp32) ln S is off by E|d| 2^-23 + 2^-22 and sum(d e)/S by E d^2 2^-23, sums of n terms by sqrt(n) 2^-24."""
    rows, classes = x.shape
    out = {"logp": [], "rank": [], "entropy": [], "top_id": [], "top_logp": [], "far": [], "far_entropy": []}
    index = torch.arange(classes)
    for r in range(rows):
        v, g = x[r].double(), -1 if given is None else int(given[r])
        bad, live = bool((~(v < math.inf)).any()), v > -math.inf
        inside = 0 <= g < classes
        far = far_h = 0.0
        if bad or not live.any():
            lp, h = (math.nan, math.nan) if bad else (-math.inf, 0.0)
            d, ls = torch.full_like(v, -math.inf), 0.0
        else:
            d = (v - v.max()) * float(torch.tensor(scale, dtype=torch.float32))
            e = torch.where(live, d, -math.inf).exp()
            s = e.sum()
            ls = float(s.log())
            de = torch.where(e > 0, d * e, 0.0)
            h = ls - float(de.sum() / s)
            lp = float(d[g]) - ls if inside else math.nan
            mean, square = float(-de.sum() / s), float(torch.where(e > 0, d * d * e, 0.0).sum() / s)
            far = 2.0 ** -24 * (64 + 8 * mean + math.sqrt(classes))
            far_h = 2.0 ** -24 * (64 + 8 * mean + 4 * square + 2 * math.sqrt(classes) * (1 + mean))
        if not inside and not bad:
            lp = math.nan
        out["logp"].append(0.0 if g < 0 else lp)
        out["rank"].append(int(((v > v[g]) | ((v == v[g]) & (index < g))).sum()) if inside and not bad else -1)
        out["entropy"].append(h)
        order = [] if bad else sorted(torch.nonzero(live).flatten().tolist(), key=lambda i: (-float(v[i]), i))[:top]
        out["top_id"].append(order + [-1] * (top - len(order)))
        out["top_logp"].append([math.nan] * top if bad else [float(d[i]) - ls for i in order] + [-math.inf] * (top - len(order)))
        out["far"].append(far)
        out["far_entropy"].append(far_h)
    return out


def assert_answer(got, ref, what=""):
    """got: tensors by name (those that were asked for)."""
    for name in ("rank", "top_id"):
        if name in got:
            assert got[name].tolist() == ref[name], (what, name, got[name].tolist(), ref[name])
    for name, far in (("logp", "far"), ("entropy", "far_entropy"), ("top_logp", "far")):
        if name not in got:
            continue
        want, have = torch.tensor(ref[name], dtype=torch.float64), got[name].double()
        limit = torch.tensor(ref[far], dtype=torch.float64)
        if want.dim() == 2:
            limit = limit[:, None]
        special = ~torch.isfinite(want)
        assert torch.equal(have[special], want[special]) or (torch.equal(torch.isnan(have[special]), torch.isnan(want[special])) and
               torch.equal(have[special & ~torch.isnan(want)], want[special & ~torch.isnan(want)])), (what, name, have, want)
        off = torch.where(special, 0.0, (have - want).abs())
        limit = limit + 2.0 ** -21 * torch.where(special, 0.0, want.abs())   # product, difference and result: four roundings of |d| + |ln S|
        assert bool((off <= limit).all()), (what, name, float((off / limit.clamp(min=1e-300)).max()), have, want)
