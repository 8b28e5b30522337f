"""What the operators around a paged key-value cache are measured on: tokens' keys and values written to pages and read back (Context.cache_write,
cache_read), the attention of one new token a sequence over them (attend_one) and of whole prompts (attend).

A case of "write" / "read":  `sequences` sequences of `shortest` to `longest` tokens, the last `share` of each written to or read from
                             pages of `page` tokens; keys and values of `kv_heads` heads of `dim` numbers, of type `x` outside and `cache` in the pages.
A case of "one":             a new token for each of `sequences` sequences, `heads` query heads over `kv_heads`, the last `window` tokens (0: all).
A case of "prompt":          `sequences` packed prompts of `shortest` to `longest` tokens, each behind `before` tokens that are there already.

Lengths go by the case alone, all else by the seed.  Pages lie in any order, as they are given out.  "e4m3" pages hold 8 bits a number and a byte a token
and head that is a power of two, 2^(byte - 127).  What a pass works on or writes is made by prepare, as a user's program has it in device memory."""
import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"fp16": 2, "bf16": 2, "fp32": 4, "e4m3": 1}
MOST_NUMBERS = 32768 * 8 * 128          # of the keys of a "write" or "read"
MOST_CACHE = 64 * 8192 * 8 * 128        # ... that an "one" has in its pages
MOST_FLOPS = 4 * 128 * 32 * 8192 * 8193 // 2    # of a "prompt"


# ---- the cases -------------------------------------------------------------------------------------
def _rows(name, op, sequences, shortest, longest, share, kv_heads, dim, page, x, cache):
    return {"name": name, "op": op, "sequences": sequences, "shortest": shortest, "longest": longest, "share": share, "kv_heads": kv_heads, "dim": dim,
            "page": page, "x": x, "cache": cache}


def _one(name, sequences, shortest, longest, heads, kv_heads, dim, page, x, cache, window=0):
    return {"name": name, "op": "one", "sequences": sequences, "shortest": shortest, "longest": longest, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "page": page, "x": x, "cache": cache, "window": window}


def _prompt(name, sequences, shortest, longest, before, heads, kv_heads, dim, x, causal=True, window=0):
    return {"name": name, "op": "prompt", "sequences": sequences, "shortest": shortest, "longest": longest, "before": before, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "x": x, "causal": causal, "window": window}


def listed():
    return [
        # a decoding batch's new tokens, one a sequence
        _rows("write-b64", "write", 64, 100, 4096, 0.0, 8, 128, 16, "bf16", "bf16"),
        # a batch of whole prompts as it is kept in 8 bits
        _rows("write-prompts-e4m3", "write", 16, 200, 4096, 1.0, 8, 128, 64, "fp16", "e4m3"),
        # a short history read back; long ones ahead of the next part of their prompts
        _rows("read-301", "read", 1, 301, 301, 1.0, 4, 64, 16, "fp16", "fp16"),
        _rows("read-b16-e4m3", "read", 16, 100, 4096, 1.0, 8, 128, 64, "bf16", "e4m3"),
        # one request, a short answer so far
        _one("one-100-b1", 1, 100, 100, 8, 8, 64, 16, "fp16", "fp16"),
        # one request with a long context
        _one("one-32001-b1", 1, 32001, 32001, 32, 8, 128, 64, "bf16", "bf16"),
        # a decoding batch of all lengths
        _one("one-8192-b64", 64, 133, 8192, 32, 8, 128, 16, "bf16", "bf16"),
        # more requests, pages of 8 bits, many queries to a key
        _one("one-4096-b200-e4m3", 200, 1, 4096, 64, 8, 128, 64, "fp16", "e4m3"),
        # a short prompt
        _prompt("prompt-77", 1, 77, 77, 0, 8, 8, 64, "fp16"),
        # what a queue held, packed; the same heads over a part of a prompt behind its longer history, looking back a window
        _prompt("prompt-b16", 16, 33, 2048, 0, 32, 8, 128, "bf16"),
        _prompt("prompt-window-b4", 4, 301, 1024, 2500, 16, 4, 96, "bf16", window=2048),
        # a long prompt: the matrix cores' work
        _prompt("prompt-8192", 1, 8192, 8192, 0, 32, 8, 128, "fp16"),
    ]


def draw(rng):
    def spread(low, high):
        return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))

    case = _draw(rng, spread)
    return {k: v for k, v in case.items() if k != "name"}


def _draw(rng, spread):
    op = rng.choice(("write", "read", "one", "one", "prompt", "prompt"))
    kv_heads, dim = rng.choice((1, 2, 4, 5, 8, 8, 16)), rng.choice((64, 64, 80, 96, 128, 128, 128, 256))
    each = rng.choice((1, 1, 2, 4, 4, 7, 8, 16))
    page, x = rng.choice((16, 16, 32, 64, 128)), rng.choice(("fp16", "bf16"))
    if op in ("write", "read"):
        longest = spread(1, 8192)
        sequences = max(1, min(spread(1, 256), MOST_NUMBERS // (longest * kv_heads * dim)))
        share = 1.0 if op == "read" else rng.choice((0.0, 0.3, 1.0))
        longest = min(longest, MOST_NUMBERS // (sequences * kv_heads * dim))
        return _rows("", op, sequences, rng.randint(1, longest), longest, share, kv_heads, dim, page, rng.choice((x, x, "fp32")), rng.choice((x, "e4m3")))
    if op == "one":
        longest = spread(1, 65536)
        sequences = max(1, min(spread(1, 256), MOST_CACHE // (longest * kv_heads * dim)))
        longest = min(longest, MOST_CACHE // (sequences * kv_heads * dim))
        window = spread(16, longest) if longest > 16 and rng.random() < 0.2 else 0
        return _one("", sequences, rng.randint(1, longest), longest, kv_heads * each, kv_heads, dim, page, x, rng.choice((x, x, "e4m3")), window)
    each = min(each, 64 // kv_heads)
    longest = spread(1, 8192)
    before = rng.choice((0, 0, 0, spread(1, 4096)))
    heads = kv_heads * each
    pairs = lambda n: n * (n + before)
    while longest > 1 and 4 * dim * heads * pairs(longest) > MOST_FLOPS * 2:
        longest //= 2
    sequences = max(1, min(spread(1, 64), MOST_FLOPS // (4 * dim * heads * pairs(longest)), 65536 // (longest + before)))
    causal = rng.random() < 0.8
    window = spread(16, longest + before) if causal and longest + before > 16 and rng.random() < 0.25 else 0
    case = _prompt("", sequences, rng.randint(1, longest), longest, before, heads, kv_heads, dim, x, causal, window)
    while work(case)["flops"] > MOST_FLOPS:
        case["longest"] //= 2
        case["shortest"] = min(case["shortest"], case["longest"])
    return case


def _lengths(case):
    """Of the sequences: from `longest` down to `shortest` in an order that mixes them."""
    n, low, high = case["sequences"], case["shortest"], case["longest"]
    return [high - (high - low) * (i * 37 % n) // max(1, n - 1) for i in range(n)]


def _new(case):
    """Tokens of each that a "write" or "read" is about."""
    return [max(1, int(n * case["share"])) for n in _lengths(case)]


# ---- what a program has in hand --------------------------------------------------------------------
class _State:
    pass


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _keys(g, dtype, *shape):
    """As projections leave them: a few loud channels, the same in every token."""
    loud = 1.0 + 9.0 * (torch.rand(shape[-2:], generator=g, device="cuda") < 0.02)
    return (torch.randn(*shape, generator=g, device="cuda") * loud).to(dtype)


def _values(g, dtype, *shape):
    return (torch.randn(*shape, generator=g, device="cuda") * (0.2 + torch.rand(*shape[:-1], 1, generator=g, device="cuda"))).to(dtype)


def _coded(x):
    """e4m3 codes and exponents of rows of numbers."""
    largest = x.float().abs().amax(-1)
    mantissa, exponent = torch.frexp(largest)                   # largest = mantissa * 2^exponent, 448 = 0.875 * 2^9
    e = (exponent - 9 + (mantissa > 0.875)).clamp(min=-127).masked_fill(largest == 0, -127)
    codes = torch.ldexp(x.float(), -e[..., None]).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def _pages(s, case, g, filled):
    """The pool of pages and the sequences' tables: a few pages more than the sequences need."""
    lengths, page = _lengths(case), case["page"]
    each = -(-case["longest"] // page)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((case["sequences"], each), -1, dtype=torch.int32, device="cuda")
    at = torch.arange(each, device="cuda") < _ints(need)[:, None]
    table[at] = order[:sum(need)]
    s.table, s.lengths = table, _ints(lengths)
    shape = (pages, case["kv_heads"], page, case["dim"])
    eight = case["cache"] == "e4m3"
    s.k_exp = s.v_exp = None
    if filled:
        s.k_cache, s.v_cache = _keys(g, torch.float16 if eight else DTYPES[case["cache"]], *shape), _values(g, torch.float16 if eight else DTYPES[case["cache"]], *shape)
        if eight:
            (s.k_cache, s.k_exp), (s.v_cache, s.v_exp) = _coded(s.k_cache), _coded(s.v_cache)
    else:
        s.k_cache, s.v_cache = (torch.zeros(shape, dtype=torch.uint8 if eight else DTYPES[case["cache"]], device="cuda") for _ in range(2))
        if eight:
            s.k_cache, s.v_cache = s.k_cache.view(torch.float8_e4m3fn), s.v_cache.view(torch.float8_e4m3fn)
            s.k_exp, s.v_exp = (torch.zeros(shape[:3], dtype=torch.uint8, device="cuda") for _ in range(2))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.op, s.handle = case["op"], None
    x = DTYPES[case["x"]]
    if s.op == "prompt":
        queries = _lengths(case)
        keys = [n + case["before"] for n in queries]
        s.first, s.first_k, s.most, s.most_k = _ints(_starts(queries)), _ints(_starts(keys)), max(queries), max(keys)
        if not case["before"]:
            s.first_k = None
        s.q = torch.randn(sum(queries), case["heads"], case["dim"], generator=g, device="cuda").to(x)
        s.k, s.v = _keys(g, x, sum(keys), case["kv_heads"], case["dim"]), _values(g, x, sum(keys), case["kv_heads"], case["dim"])
        s.y, s.lse = torch.zeros_like(s.q), torch.zeros(s.q.shape[:2], device="cuda")
        s.causal, s.window, s.scale = case["causal"], case["window"], 1.0 / math.sqrt(case["dim"])
        return s
    _pages(s, case, g, s.op != "write")
    if s.op == "one":
        s.q = torch.randn(case["sequences"], case["heads"], case["dim"], generator=g, device="cuda").to(x)
        s.y, s.lse = torch.zeros_like(s.q), torch.zeros(s.q.shape[:2], device="cuda")
        s.window, s.scale = case["window"], 1.0 / math.sqrt(case["dim"])
        s.workspace = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
        return s
    first = _starts(_new(case))
    s.first = _ints(first)
    shape = (first[-1], case["kv_heads"], case["dim"])
    s.k, s.v = (_keys(g, x, *shape), _values(g, x, *shape)) if s.op == "write" else (torch.zeros(shape, dtype=x, device="cuda") for _ in range(2))
    return s


# ---- the plain forms -------------------------------------------------------------------------------
def _places(s):
    """Page and place in it of every new token."""
    token = torch.arange(s.k.shape[0], device="cuda", dtype=torch.int32)
    sequence = torch.searchsorted(s.first, token, right=True) - 1
    position = token - s.first[sequence + 1] + s.lengths[sequence]
    page = s.k_cache.shape[2]
    return s.table[sequence, position // page].long(), position.long() % page


def _plain_write(s):
    page, at = _places(s)
    for new, cache, exps in ((s.k, s.k_cache, s.k_exp), (s.v, s.v_cache, s.v_exp)):
        if exps is None:
            cache[page, :, at] = new.to(cache.dtype)
        else:
            codes, e = _coded(new)
            cache.view(torch.uint8)[page, :, at] = codes.view(torch.uint8)
            exps[page, :, at] = e
    return _written(s)


def _written(s):
    out = {"k_cache": s.k_cache, "v_cache": s.v_cache}
    if s.k_exp is not None:
        out["k_exp"], out["v_exp"] = s.k_exp, s.v_exp
    return out


def _decoded(cache, exps, *at):
    """Numbers of cache[at] in 32 bits."""
    if exps is None:
        return cache[at].float()
    return torch.ldexp(cache.view(torch.uint8)[at].view(torch.float8_e4m3fn).float(), exps[at].int()[..., None] - 127)


def _plain_read(s):
    page, at = _places(s)
    every = slice(None)
    return {"k": _decoded(s.k_cache, s.k_exp, page, every, at).to(s.k.dtype), "v": _decoded(s.v_cache, s.v_exp, page, every, at).to(s.v.dtype)}


def _softmax_times(scores, seen, v):
    """Rows of softmax(scores where seen) times v, and the logs of their sums; 0 and -inf of rows that see nothing."""
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(scores - top)
    total = e.sum(-1, keepdim=True)
    y = torch.matmul(e, v) / torch.where(total > 0, total, 1.0)
    return y, (top + torch.log(total))[..., 0]


def _plain_one(s):
    sequences, heads, dim = s.q.shape
    kv_heads, page = s.k_cache.shape[1:3]
    table = s.table.clamp(min=0).long()
    tokens = table.shape[1] * page
    gather = lambda cache, exps: _decoded(cache, exps, table).transpose(1, 2).reshape(sequences, kv_heads, tokens, dim)
    k, v = gather(s.k_cache, s.k_exp), gather(s.v_cache, s.v_exp)
    scores = torch.matmul(s.q.float().view(sequences, kv_heads, heads // kv_heads, dim), k.transpose(2, 3)) * s.scale
    at = torch.arange(tokens, device="cuda")
    seen = at < s.lengths[:, None]
    if s.window:
        seen &= at >= s.lengths[:, None] - s.window
    y, lse = _softmax_times(scores, seen[:, None, None], v)
    return {"y": y.reshape(s.q.shape).to(s.y.dtype), "lse": lse.reshape(sequences, heads)}


def _padded(x, first, most):
    """[sequences][heads][most][dim] of packed rows, in 32 bits, and which of them are rows."""
    at = first[:-1, None] + torch.arange(most, device="cuda")
    real = at < first[1:, None]
    return (x[at.clamp(max=x.shape[0] - 1).long()].float() * real[..., None, None]).transpose(1, 2), real


def _plain_prompt(s):
    first_k = s.first if s.first_k is None else s.first_k
    q, rows = _padded(s.q, s.first, s.most)
    k, keys = _padded(s.k, first_k, s.most_k)
    v, _ = _padded(s.v, first_k, s.most_k)
    sequences, heads, most, dim = q.shape
    kv_heads = k.shape[1]
    q = q.reshape(sequences, kv_heads, heads // kv_heads * most, dim)
    scores = (torch.matmul(q, k.transpose(2, 3).contiguous()) * s.scale).view(sequences, kv_heads, heads // kv_heads, most, s.most_k)
    seen = keys[:, None]
    if s.causal:
        behind = (first_k[1:] - first_k[:-1] - s.first[1:] + s.first[:-1])[:, None, None]
        ago = torch.arange(most, device="cuda")[:, None] + behind - torch.arange(s.most_k, device="cuda")     # how long before the query the key is
        seen = seen & (ago >= 0) & ((ago < s.window) if s.window else True)
    y, lse = _softmax_times(scores.flatten(2, 3), seen[:, None, None].expand(scores.shape).flatten(2, 3), v)
    y, lse = y.view(sequences, heads, most, dim).transpose(1, 2)[rows], lse.view(sequences, heads, most).transpose(1, 2)[rows]
    return {"y": y.to(s.y.dtype), "lse": lse}


# ---- one pass --------------------------------------------------------------------------------------
_contexts = []


def _context():
    """The worker's context: one per process, as one worker has."""
    if not _contexts:
        from paper_2006_02464_amd.binding import Context
        _contexts.append(Context(workspace_bytes=16 << 20, io_bytes=1 << 20, weight_pool_bytes=16 << 20, load_staging_bytes=1 << 20))
    return _contexts[0]


def _own(s):
    ctx, stream = _context(), torch.cuda.current_stream()
    if s.op == "prompt":
        ctx.attend(s.q, s.k, s.v, s.y, s.first, first_k=s.first_k, causal=s.causal, window=s.window, scale=s.scale, lse=s.lse, stream=stream)
        return {"y": s.y, "lse": s.lse}
    if s.handle is None:        # kept beside the pool of pages that it names, as a program does
        s.handle = ctx.cache(s.k_cache, s.v_cache, k_exp=s.k_exp, v_exp=s.v_exp)
    if s.op == "one":
        ctx.attend_one(s.q, s.handle, s.table, s.lengths, s.y, window=s.window, scale=s.scale, lse=s.lse, workspace=s.workspace, stream=stream)
        return {"y": s.y, "lse": s.lse}
    if s.op == "write":
        ctx.cache_write(s.k, s.v, s.handle, s.table, s.lengths, first=s.first, stream=stream)
        return _written(s)
    ctx.cache_read(s.handle, s.table, s.lengths, s.k, s.v, first=s.first, stream=stream)
    return {"k": s.k, "v": s.v}


def run(s):
    if own:
        return _own(s)
    return {"write": _plain_write, "read": _plain_read, "one": _plain_one, "prompt": _plain_prompt}[s.op](s)


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    """write, read: every number of the tokens in question read once and written once, with its exponents.
    one: keys and values that are looked at read once, queries and results; a multiply and an add a number and query head.
    prompt: queries, keys, values and results once; two products a query and key that it sees."""
    heads, dim, x = case["kv_heads"], case["dim"], SIZE[case["x"]]
    if case["op"] == "prompt":
        heads, window = case["heads"], case["window"]
        pairs = tokens = keys = 0
        for n in _lengths(case):
            m = n + case["before"]
            tokens, keys = tokens + n, keys + m
            if not case["causal"]:
                pairs += n * m
                continue
            full = n * case["before"] + n * (n + 1) // 2            # query i sees before + i + 1 keys
            over = max(0, min(n, m - window)) if window else 0      # ... the last `over` of them only `window`
            pairs += full - (over * (m - window) - over * (over - 1) // 2)
        return {"bytes": (2 * tokens * heads + 2 * keys * case["kv_heads"]) * dim * x + 4 * tokens * heads, "flops": 4 * dim * heads * pairs}
    kept = 2 * heads * (dim * SIZE[case["cache"]] + (case["cache"] == "e4m3"))      # bytes of a token in the pages
    if case["op"] == "one":
        seen = sum(min(n, case["window"]) if case["window"] else n for n in _lengths(case))
        rows = case["sequences"] * case["heads"]
        return {"bytes": seen * kept + rows * (2 * dim * x + 4), "flops": 4 * seen * case["heads"] * dim}
    tokens = sum(_new(case))
    return {"bytes": tokens * (kept + 2 * heads * dim * x), "flops": 2 * tokens * heads * dim}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _attention64(q, k, v, scale, seen):
    """[heads][queries][dim] over [kv_heads][keys][dim]."""
    each = q.shape[0] // k.shape[0]
    y, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for h in range(q.shape[0]):
        for a in range(0, q.shape[1], 2048):
            score = torch.matmul(q[h, a:a + 2048], k[h // each].t().contiguous()) * scale
            score = score.masked_fill(~seen[a:a + 2048], -math.inf)
            lse[h, a:a + 2048] = torch.logsumexp(score, 1)
            y[h, a:a + 2048] = torch.matmul(torch.exp(score - lse[h, a:a + 2048, None]).nan_to_num(0.0), v[h // each])
    return y, lse


def _history64(s, i, n):
    """Keys and values of the n tokens of sequence i in the pages: [kv_heads][n][dim]."""
    page = s.k_cache.shape[2]
    at = s.table[i, :-(-n // page)].long()

    def numbers(cache, exps):
        x = cache[at].double() if exps is None else cache.view(torch.uint8)[at].view(torch.float8_e4m3fn).double() * torch.exp2(exps[at].double() - 127)[..., None]
        return x.permute(1, 0, 2, 3).flatten(1, 2)[:, :n]
    return numbers(s.k_cache, s.k_exp), numbers(s.v_cache, s.v_exp)


def exact(case, seed):
    s = prepare(case, seed)
    lengths = _lengths(case)
    if s.op == "prompt":
        y, lse = s.q.double(), torch.zeros(s.q.shape[:2], dtype=torch.float64, device="cuda")
        first, first_k = _starts(lengths), _starts([n + case["before"] for n in lengths])
        for i, n in enumerate(lengths):
            a, b, m = first[i], first_k[i], n + case["before"]
            seen = torch.ones(n, m, dtype=torch.bool, device="cuda")
            if s.causal:
                seen = seen.tril(m - n)
            if s.window:
                seen &= ~torch.ones_like(seen).tril(m - n - s.window)
            out = _attention64(s.q[a:a + n].double().transpose(0, 1), s.k[b:b + m].double().transpose(0, 1), s.v[b:b + m].double().transpose(0, 1).contiguous(), s.scale, seen)
            y[a:a + n], lse[a:a + n] = out[0].transpose(0, 1), out[1].t()
        return {"y": y, "lse": lse}
    if s.op == "one":
        y, lse = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda"), torch.zeros(s.q.shape[:2], dtype=torch.float64, device="cuda")
        for i, n in enumerate(lengths):
            k, v = _history64(s, i, n)
            from_ = max(0, n - s.window) if s.window else 0
            k, v = k[:, from_:], v[:, from_:]
            kv_heads, dim = k.shape[0], k.shape[2]
            score = torch.matmul(s.q[i].double().view(kv_heads, -1, dim), k.transpose(1, 2).contiguous()) * s.scale
            lse[i] = torch.logsumexp(score, 2).flatten()
            y[i] = torch.matmul(torch.softmax(score, 2), v.contiguous()).reshape(-1, dim)
        return {"y": y, "lse": lse}
    new, first, page = _new(case), _starts(_new(case)), case["page"]
    if s.op == "read":
        k, v = (torch.zeros(s.k.shape, dtype=torch.float64, device="cuda") for _ in range(2))
        for i, n in enumerate(lengths):
            hk, hv = _history64(s, i, n)
            k[first[i]:first[i + 1]], v[first[i]:first[i + 1]] = hk[:, n - new[i]:].transpose(0, 1), hv[:, n - new[i]:].transpose(0, 1)
        return {"k": k, "v": v}
    out = {}
    for name, x in (("k_cache", s.k.double()), ("v_cache", s.v.double())):
        to = torch.zeros(s.k_cache.shape, dtype=torch.float64, device="cuda")
        if s.k_exp is not None:
            x = x * torch.exp2(-torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448.0)).clamp(min=-127))
        for i, n in enumerate(lengths):
            at = torch.arange(n - new[i], n, device="cuda")
            to[s.table[i].long()[at // page], :, at % page] = x[first[i]:first[i + 1]]
        out[name] = to
    if s.k_exp is not None:
        out["k_exp"] = out["v_exp"] = None
    return out
