"""What the operators at the end of a network are measured on: the fully connected layer over 4-bit weights (Context.fc4) and the
answer over its logits (Context.answer), over the range of sizes and types that classifiers and vocabularies have.

A case of "fc4":    rows x cin activations of type `x`, cout rows of 4-bit weights with one scale (and, with `zeros`, one zero
                    point) for each `group` of inputs, results of type `y`.
A case of "answer": `rows` rows of `classes` logits of type `x`; of each, the log probability and rank of a given class, the entropy
                    and the `top` likeliest classes.  `banned` is the share of classes that a mask has taken out (-inf).

Whatever tensors a pass works on or writes are made by prepare, as a user's program has them in device memory."""
import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
MOST_MACS = 512 * 4096 * 4096       # of one fc4 pass
MOST_WEIGHTS = 8192 * 32001
MOST_LOGITS = 2048 * 32000


# ---- the cases -------------------------------------------------------------------------------------
def _fc4(name, rows, cin, cout, group, x, y, zeros=False, features=False):
    return {"name": name, "op": "fc4", "rows": rows, "cin": cin, "cout": cout, "group": group, "x": x, "y": y, "zeros": zeros, "features": features}


def _answer(name, rows, classes, top, x, temperature=1.0, banned=0.0):
    return {"name": name, "op": "answer", "rows": rows, "classes": classes, "top": top, "x": x, "temperature": temperature, "banned": banned}


def listed():
    return [
        # the classifiers of the benchmark's networks: one image of the smallest, a throughput batch; pooled features in fp32
        _fc4("fc4-512x1000-b1", 1, 512, 1000, 64, "fp32", "fp32", features=True),
        _fc4("fc4-2048x1000-b16", 16, 2048, 1000, 128, "fp32", "fp32", features=True),
        # one token or request through a square layer
        _fc4("fc4-4096x4096-b1", 1, 4096, 4096, 128, "fp16", "fp16"),
        # the widest head, one request, an odd number of classes: nothing but reading weights
        _fc4("fc4-8192x32001-b1", 1, 8192, 32001, 128, "bf16", "fp32"),
        # whatever a queue held, odd sizes, the finest groups
        _fc4("fc4-1000x777-b5", 5, 1000, 777, 32, "bf16", "bf16", zeros=True),
        # a decoding batch
        _fc4("fc4-4096x16384-b64", 64, 4096, 16384, 64, "fp16", "fp16", zeros=True),
        # a whole prompt: the matrix cores' work
        _fc4("fc4-4096x4096-b512", 512, 4096, 4096, 128, "bf16", "bf16"),
        # the answer of one image; of a batch of them
        _answer("answer-1000-b1", 1, 1000, 5, "fp32"),
        _answer("answer-1000-b16", 16, 1000, 5, "fp32"),
        # one token from a large vocabulary, some of it banned
        _answer("answer-131072-b1", 1, 131072, 20, "fp16", temperature=0.7, banned=0.3),
        # a decoding batch, an odd vocabulary
        _answer("answer-50001-b64", 64, 50001, 10, "bf16"),
        # scoring given text: no alternatives asked for
        _answer("answer-32000-b2048", 2048, 32000, 0, "fp32"),
    ]


def draw(rng):
    def spread(low, high):
        return min(high, max(low, int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))))

    if rng.random() < 0.55:
        rows, cin, cout = spread(1, 512), spread(16, 8192), spread(8, 32001)
        group = rng.choice((32, 64, 128, 128, 256))
        if rng.random() < 0.7:
            cin = max(group, cin // group * group)      # the usual: whole groups
        cout = min(cout, MOST_WEIGHTS // cin, MOST_MACS // cin)
        rows = max(1, min(rows, MOST_MACS // (cin * cout)))
        x = rng.choice(("fp16", "bf16", "fp32"))
        y = rng.choice((x, "fp32"))
        return {k: v for k, v in _fc4("", rows, cin, cout, group, x, y, rng.random() < 0.4, x == "fp32" and rng.random() < 0.5).items() if k != "name"}
    classes = spread(10, 131072)
    rows = max(1, min(spread(1, 2048), MOST_LOGITS // classes))
    case = _answer("", rows, classes, min(classes, rng.choice((0, 1, 5, 10, 20, 50))), rng.choice(("fp16", "bf16", "fp32")),
                   rng.choice((1.0, 1.0, 0.7, 1.3)), rng.choice((0.0, 0.0, 0.3, 0.9)))
    return {k: v for k, v in case.items() if k != "name"}


# ---- what a program has in hand --------------------------------------------------------------------
class _State:
    pass


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = _State()
    s.op = case["op"]
    if s.op == "fc4":
        rows, cin, cout, group = case["rows"], case["cin"], case["cout"], case["group"]
        groups = -(-cin // group)
        x = torch.randn(rows, cin, generator=g, device="cuda")
        if case["features"]:
            x = x.abs() * 0.8                                   # averages of activations behind a ReLU
        else:
            x = x * (1.0 + 7.0 * (torch.rand(cin, generator=g, device="cuda") < 0.01))     # a few loud channels
        s.x = x.to(DTYPES[case["x"]])
        q = torch.randn(cout, cin + cin % 2, generator=g, device="cuda").mul_(2.7).add_(8.0).round_().clamp_(0, 15).to(torch.uint8)
        if cin % 2:
            q[:, -1] = 0
        s.q = q[:, 0::2] | (q[:, 1::2] << 4)
        del q
        half = torch.bfloat16 if case["x"] == "bf16" else torch.float16
        s.scales = ((0.5 + torch.rand(cout, groups, generator=g, device="cuda")) * (0.35 / math.sqrt(cin))).to(half)
        s.zeros = torch.randint(5, 12, (cout, groups), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
        s.bias = torch.randn(cout, generator=g, device="cuda") * 0.1
        s.group = group
        s.y = torch.zeros(rows, cout, dtype=DTYPES[case["y"]], device="cuda")
    else:
        rows, classes, top = case["rows"], case["classes"], case["top"]
        x = torch.randn(rows, classes, generator=g, device="cuda") * 2.5
        given = torch.randint(0, classes, (rows,), generator=g, device="cuda")
        x[torch.arange(rows, device="cuda"), given] += 6.0 * torch.rand(rows, generator=g, device="cuda")
        if case["banned"] > 0:
            keep = torch.rand(classes, generator=g, device="cuda") >= case["banned"]
            keep[0] = True
            x = torch.where(keep, x, -math.inf)
        given[3::17] = -1                                       # rows of a padded batch: nothing given
        s.logits, s.given, s.top, s.scale = x.to(DTYPES[case["x"]]), given.to(torch.int32), top, 1.0 / case["temperature"]
        s.logp, s.entropy = (torch.zeros(rows, device="cuda") for _ in range(2))
        s.rank = torch.zeros(rows, dtype=torch.int32, device="cuda")
        s.top_id, s.top_logp = torch.zeros(rows, top, dtype=torch.int32, device="cuda"), torch.zeros(rows, top, device="cuda")
        s.workspace = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms -------------------------------------------------------------------------------
def _plain_fc4(s):
    cin = s.x.shape[1]
    q = torch.stack((s.q & 15, s.q >> 4), 2).flatten(1)[:, :cin].float()
    wide = lambda v: v.float().repeat_interleave(s.group, 1)[:, :cin]
    w = (q - (wide(s.zeros) if s.zeros is not None else 8.0)) * wide(s.scales)
    return {"y": (s.x.float() @ w.t() + s.bias).to(s.y.dtype)}


def _plain_answer(s):
    x = s.logits.float() + 0.0
    rows, classes = x.shape
    index = torch.arange(classes, device=x.device)
    top = x.amax(1, keepdim=True)
    d = (x - top) * s.scale
    e = torch.exp(d)
    total = e.sum(1)
    log_total = torch.log(total)
    entropy = log_total - torch.where(e > 0, e * d, 0.0).sum(1) / total
    some, g = s.given >= 0, s.given.clamp(min=0).long()[:, None]
    xg = x.gather(1, g)
    rank = torch.where(some, ((x > xg) | ((x == xg) & (index < g))).sum(1), -1).to(torch.int32)
    logp = torch.where(some, d.gather(1, g)[:, 0] - log_total, 0.0)
    out = {"logp": logp, "rank": rank, "entropy": entropy}
    if s.top:
        bits = x.view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7fffffff)).long() * (1 << 32) + ((1 << 32) - 1 - index)      # ties: the lowest index is the largest
        at = order.topk(s.top, 1).indices
        value = d.gather(1, at) - log_total[:, None]
        out["top_id"], out["top_logp"] = torch.where(value > -math.inf, at, -1).to(torch.int32), value
    return out


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
    if s.op == "fc4":
        ctx.fc4(s.x, s.q, s.scales, s.y, s.group, zeros=s.zeros, bias=s.bias, stream=stream)
        return {"y": s.y}
    ctx.answer(s.logits, s.given, logp=s.logp, rank=s.rank, entropy=s.entropy, top_id=s.top_id if s.top else None,
               top_logp=s.top_logp if s.top else None, scale=s.scale, workspace=s.workspace, stream=stream)
    out = {"logp": s.logp, "rank": s.rank, "entropy": s.entropy}
    if s.top:
        out["top_id"], out["top_logp"] = s.top_id, s.top_logp
    return out


def run(s):
    if own:
        return _own(s)
    return _plain_fc4(s) if s.op == "fc4" else _plain_answer(s)


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    """fc4: activations, weights, scales, zero points and biases read once, results written; a multiply and an add for every weight and row.
    answer: logits read once, answers written; six operations a logit (difference, scale, exponential, two sums, comparison)."""
    size = {"fp16": 2, "bf16": 2, "fp32": 4}
    rows = case["rows"]
    if case["op"] == "fc4":
        cin, cout, groups = case["cin"], case["cout"], -(-case["cin"] // case["group"])
        weights = cout * (-(-cin // 2) + groups * (3 if case["zeros"] else 2) + 4)
        return {"bytes": rows * cin * size[case["x"]] + weights + rows * cout * size[case["y"]], "flops": 2 * rows * cin * cout}
    return {"bytes": rows * case["classes"] * size[case["x"]] + rows * (16 + 8 * case["top"]), "flops": 6 * rows * case["classes"]}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if s.op == "fc4":
        rows, cin = s.x.shape
        cout = s.q.shape[0]
        y = s.bias.double().repeat(rows, 1)
        for j in range(s.scales.shape[1]):                      # group by group: y += s_j * (x_j q_j^T - z_j sum x_j)
            k0, k1 = j * s.group, min(cin, (j + 1) * s.group)
            part = s.q[:, k0 // 2:(k1 + 1) // 2]
            q = torch.empty(cout, part.shape[1] * 2, dtype=torch.float64, device="cuda")
            q[:, 0::2], q[:, 1::2] = part.remainder(16), part.div(16, rounding_mode="floor")
            q = q[:, :k1 - k0] - (8.0 if s.zeros is None else s.zeros[:, j:j + 1].double())
            y += torch.matmul(s.x[:, k0:k1].double(), q.t().contiguous()) * s.scales[:, j].double()
        return {"y": y}
    x = s.logits.double() * s.scale
    lse = torch.logsumexp(x, 1)
    logp = x - lse[:, None]
    p = logp.exp()
    given = s.given.long()
    out = {"logp": torch.where(given < 0, 0.0, logp.gather(1, given.clamp(min=0)[:, None])[:, 0]), "rank": None,
           "entropy": -torch.where(p > 0, p * logp, 0.0).sum(1)}
    if s.top:
        out["top_id"], out["top_logp"] = None, logp.topk(s.top, 1).values
    return out
