"""Plain 64-bit forms of the paged cache and of the attentions, and the bounds that their tests use."""
import math

import torch

F16, BF16, F32, E4M3 = torch.float16, torch.bfloat16, torch.float32, torch.float8_e4m3fn
HALF_STEP = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}
SMALLEST = {F16: 2.0 ** -25, BF16: 2.0 ** -134, F32: 2.0 ** -150}   # half of the smallest step
INF, NAN = float("inf"), float("nan")


# ---- the cache -------------------------------------------------------------------------------------
def coded(x):
    """(e4m3 codes as bytes, exponents) of the rows of x, number by number."""
    x = x.double()
    finite = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    e = torch.full(finite.shape, -127, dtype=torch.int64)
    for _ in range(256):                                    # the least e from -127 on with finite <= 448 * 2^e
        e += (finite > 448.0 * torch.exp2(e.double())).long()
    y = torch.where(x.isfinite(), x, NAN) * torch.exp2(-e.double())[..., None]
    m = y.abs()
    step = torch.exp2(torch.floor(torch.log2(m.clamp(min=2.0 ** -6))) - 3)      # 2^-9 below 2^-6
    low = torch.floor(m / step)
    rest = m / step - low
    n = low + ((rest > 0.5) | ((rest == 0.5) & (low % 2 == 1))).double()        # ties to even
    value = torch.copysign(n * step, y)
    codes = torch.where(y.isnan(), NAN, value).float().to(E4M3)                 # exact: they are e4m3 numbers
    assert torch.equal(codes.double()[~y.isnan()], value[~y.isnan()])
    return codes.view(torch.uint8), (e + 127).to(torch.uint8)


def decoded(codes, exponents):
    return codes.view(E4M3).double() * torch.exp2(exponents.double() - 127)[..., None]


class Pages:
    """A pool of pages on the CPU and the sequences' tables, pages given out in any order; what no sequence has is NaN."""

    def __init__(self, lengths, kv_heads, page, dim, dtype, seed=0, table_pages=None, spare=2):
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // page) for n in lengths]
        self.pages, self.page, self.dtype, self.lengths = sum(need) + spare, page, dtype, list(lengths)
        each = max(need + [1]) if table_pages is None else table_pages
        order = torch.randperm(self.pages, generator=g)
        self.table = torch.full((len(lengths), each), -1, dtype=torch.int32)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n].to(torch.int32)[:each]
            at += n
        shape = (self.pages, kv_heads, page, dim)
        self.k_exp = self.v_exp = None
        if dtype == E4M3:
            self.k, self.v = (torch.full(shape, 0x7f, dtype=torch.uint8) for _ in range(2))
            self.k_exp, self.v_exp = (torch.full(shape[:3], 255, dtype=torch.uint8) for _ in range(2))
        else:
            self.k, self.v = (torch.full(shape, NAN, dtype=dtype) for _ in range(2))

    def places(self, i, a, b):
        """(sequence's tokens, pages, places) of tokens a..b - 1 that have one."""
        a = max(a, 0)
        t = torch.arange(a, max(a, min(b, self.table.shape[1] * self.page)))
        page = self.table[i].long()[t // self.page]
        ok = (page >= 0) & (page < self.pages)
        return t[ok], page[ok], t[ok] % self.page

    def write(self, i, k, v, end):
        """Rows as the last tokens of sequence i, that has `end` tokens with them."""
        begin = end - k.shape[0]
        t, page, at = self.places(i, begin, end)
        for new, to, exps in ((k, self.k, self.k_exp), (v, self.v, self.v_exp)):
            if exps is None:
                to[page, :, at] = new[t - begin].to(to.dtype)
            else:
                to[page, :, at], exps[page, :, at] = coded(new[t - begin])

    def read(self, i, a, b):
        """Tokens a..b - 1 of sequence i in 64 bits, [tokens][kv_heads][dim] of keys and of values, 0 where there are none, and where there are some."""
        t, page, at = self.places(i, a, b)
        out = []
        for x, exps in ((self.k, self.k_exp), (self.v, self.v_exp)):
            to = torch.zeros(b - a, x.shape[1], x.shape[3], dtype=torch.float64)
            to[t - a] = x[page, :, at].double() if exps is None else decoded(x[page, :, at], exps[page, :, at])
            out.append(to)
        there = torch.zeros(b - a, dtype=torch.bool)
        there[t - a] = True
        return out[0], out[1], there

    def fill(self, seed=1, spread=1.0, loud=True):
        """Every sequence's tokens, as projections leave them."""
        g = torch.Generator().manual_seed(seed)
        heads, dim = self.k.shape[1], self.k.shape[3]
        by = 1.0 + 9.0 * (torch.rand(heads, dim, generator=g) < 0.03) if loud else 1.0
        x = F16 if self.dtype == E4M3 else self.dtype
        for i, n in enumerate(self.lengths):
            if n > 0:
                self.write(i, (torch.randn(n, heads, dim, generator=g) * by * spread).to(x), torch.randn(n, heads, dim, generator=g).to(x), n)
        return self

    def cuda(self, ctx, layout="head first"):
        """The handle of a copy on the GPU, and the copy: pages [heads][page] or [page][heads]."""
        def to(x, last):
            if x is None:
                return None
            if layout == "token first":
                return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
            return x.cuda()
        k, v, ke, ve = to(self.k, 1), to(self.v, 1), to(self.k_exp, 0), to(self.v_exp, 0)
        if self.dtype == E4M3:
            k, v = k.view(E4M3), v.view(E4M3)
        return ctx.cache(k, v, k_exp=ke, v_exp=ve), (k, v, ke, ve)


# ---- attention -------------------------------------------------------------------------------------
def attention(q, k, v, scale, seen, p_step):
    """softmax(scale q k^T where seen) v of [queries][heads][dim] over [keys][kv_heads][dim] in 64 bits: y, lse and the bounds of what a kernel gives before y's own rounding.

    A score's fp32 sum of dim products is off by (2 sqrt(dim) + 8) 2^-24 of A = scale sum |q k| (roundings that add up like chance does, but for rare luck), it and the maximum are
    scaled and subtracted in fp32: 2^-22 of their sizes, and exponentials have 2^-22: a weight is off by `far` of itself, and y, a quotient of two sums of weights, by twice
    that of sum p |v|; sums of n of them add (2 sqrt(n) + 8) 2^-24 each.  Weights go into the second product in fewer bits, p_step of each (and 2^-25 of the largest where fp16 ends)."""
    n, heads, dim = q.shape
    each = heads // k.shape[1]
    y, lse = torch.zeros(n, heads, dim, dtype=torch.float64), torch.full((n, heads), -INF, dtype=torch.float64)
    off_y, off_lse = torch.zeros_like(y), torch.zeros_like(lse)
    for h in range(heads):
        kh, vh, qh = k[:, h // each].double(), v[:, h // each].double(), q[:, h].double()
        kh0, vh0 = kh.nan_to_num(0.0, 0.0, 0.0), vh.nan_to_num(0.0, 0.0, 0.0)
        if k.shape[0] == 0:
            continue
        s = torch.where(seen, scale * (qh @ kh.t()), -INF)
        a = torch.where(seen, abs(scale) * (qh.nan_to_num(0.0).abs() @ kh0.abs().t()), 0.0).amax(1)
        top = s.amax(1)
        some = top > -INF
        e = torch.exp(s - torch.where(some, top, 0.0)[:, None])
        total = e.sum(1)
        p = e / torch.where(some, total, 1.0)[:, None]
        if bool(torch.isfinite(vh).all()):
            y[:, h] = p @ vh
        else:                                               # 0 times what is not seen is nothing
            y[:, h] = torch.where(seen[..., None], p[..., None] * vh, 0.0).sum(1)
        lse[:, h] = torch.where(some | top.isnan(), top + torch.log(total), -INF)
        far = (2 * math.sqrt(dim) + 8) * 2.0 ** -24 * a + 2.0 ** -22 * (2 * a + 4)
        sums = (2 * math.sqrt(k.shape[0]) + 8) * 2.0 ** -24
        size = p.nan_to_num(0.0) @ vh0.abs()
        few = 2.0 ** -25 / torch.where(some, total, 1.0)[:, None] * (seen.double() @ vh0.abs()) if p_step != HALF_STEP[BF16] else 0.0
        off_y[:, h] = (2 * far + 2 * sums + p_step)[:, None] * size + few
        off_lse[:, h] = far + sums + 2.0 ** -22 * (1 + lse[:, h].nan_to_num(0.0, 0.0, 0.0).abs())
    return y, lse, off_y, off_lse


def seen_causal(n, m, causal=True, window=0):
    ago = torch.arange(n)[:, None] + (m - n) - torch.arange(m)
    if not causal:
        return torch.ones(n, m, dtype=torch.bool)
    return (ago >= 0) & ((ago < window) if window else torch.ones_like(ago, dtype=torch.bool))


def assert_attention(y, lse, ref, what=""):
    ry, rl, off_y, off_l = ref
    same = lambda got, want: bool((got.isnan() == want.isnan()).all())
    assert same(y.double(), ry), (what, "NaN of y")
    fine = ~ry.isnan()
    bound = off_y * 1.001 + HALF_STEP[y.dtype] * (ry.abs() + off_y) + SMALLEST[y.dtype]
    worst = ((y.double() - ry).abs() / bound)[fine]
    assert worst.numel() == 0 or bool((worst <= 1).all()), (what, "y", float(worst.max()))
    if lse is None:
        return
    assert same(lse.double(), rl), (what, "NaN of lse")
    assert torch.equal(lse == -INF, rl == -INF), (what, "empty rows")
    fine = rl.isfinite()
    worst = ((lse.double() - rl).abs() / off_l)[fine]
    assert worst.numel() == 0 or bool((worst <= 1).all()), (what, "lse", float(worst.max()))
