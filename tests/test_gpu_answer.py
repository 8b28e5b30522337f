"""cw_answer against 64 bits: sizes from one on, types, masks that leave little or nothing, ties, orders that selection finds hard,
strides, streams and graphs, and the chain of cw_fc4 and cw_answer."""
import math

import pytest
import torch

import paper_2006_02464_amd as cw
from operator_refs import answer_ref, assert_answer, assert_fc4, fc4_data, fc4_ref

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    c = cw.Context(workspace_bytes=16 << 20, io_bytes=1 << 20, weight_pool_bytes=16 << 20, load_staging_bytes=1 << 20)
    yield c
    c.destroy()


def outputs(rows, top, fill=-7):
    out = {k: torch.full((rows,), float(fill), device="cuda") for k in ("logp", "entropy")}
    out["rank"] = torch.full((rows,), fill, dtype=torch.int32, device="cuda")
    if top:
        out["top_id"], out["top_logp"] = torch.full((rows, top), fill, dtype=torch.int32, device="cuda"), torch.full((rows, top), float(fill), device="cuda")
    return out


def call(ctx, x, given, top, scale=1.0, workspace=None, out=None, stream=None):
    out = outputs(x.shape[0], top) if out is None else out
    ctx.answer(x, given, scale=scale, workspace=workspace, stream=torch.cuda.current_stream() if stream is None else stream, **out)
    return out


def new_workspace(ctx):
    return torch.zeros(ctx.answer_workspace_bytes(), dtype=torch.uint8, device="cuda")


def check(ctx, x, given, top, scale=1.0, what=""):
    """With and without a workspace; x, given on the CPU."""
    ref = answer_ref(x, given, top, scale)
    xd, gd = x.cuda(), None if given is None else given.cuda()
    workspace = new_workspace(ctx)
    for ws in (None, workspace, workspace):
        got = {k: v.cpu() for k, v in call(ctx, xd, gd, top, scale, ws).items()}
        assert_answer(got, ref, (what, ws is not None))
    assert not bool(workspace[:cw.CW_ANSWER_COUNTERS].any())


def logits(rows, classes, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, classes, generator=g) * spread).to(dtype), torch.randint(0, classes, (rows,), generator=g, dtype=torch.int32)


SIZES = [(1, 1, 1), (2, 2, 2), (1, 3, 5), (3, 10, 3), (5, 63, 64), (4, 64, 64), (2, 65, 10), (3, 127, 1), (2, 255, 20), (2, 256, 5), (3, 257, 64), (1, 1000, 5), (16, 1000, 5),
         (300, 1000, 3), (2, 1023, 8), (3, 1025, 8), (2, 2047, 50), (1, 4096, 64), (1, 4097, 20), (2, 8191, 0), (2, 10007, 33), (1, 32768, 64), (3, 32769, 17), (1, 65537, 10),
         (1, 131072, 20), (70, 5003, 10), (260, 517, 64), (1, 200001, 64)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_sizes(ctx, size, dtype):
    rows, classes, top = size
    x, given = logits(rows, classes, dtype, sum(size))
    if rows > 2:
        given[1] = -1
    check(ctx, x, given, top, (1.0, 0.7, 1.9)[rows % 3])


@pytest.mark.parametrize("classes", [7, 1000, 9000, 70001])
def test_masks(ctx, classes):
    """Masked classes take no part; a row of nothing, one class left, fewer than asked for, the type's lowest value in the place of -inf."""
    for dtype in (F16, BF16, F32):
        x, given = logits(12, classes, dtype, classes)
        g = torch.Generator().manual_seed(1)
        x[1] = torch.where(torch.rand(classes, generator=g) < 0.9, -INF, x[1])
        x[2] = -INF
        x[3] = -INF
        x[3, classes // 2] = 2.0
        given[3] = classes // 2
        x[4] = -INF
        x[4, ::max(2, classes // 4)] = 1.0
        x[5, given[5]] = -INF
        low = torch.finfo(dtype).min
        x[6] = low
        x[7, 1:] = low
        x[8] = -INF
        x[8, -1] = low
        x[9, :-1] = -INF
        given[10] = -3
        x[11] = torch.finfo(dtype).max
        check(ctx, x, given, min(64, classes + 2), what=dtype)


@pytest.mark.parametrize("classes", [7, 1000, 9000, 70001])
@pytest.mark.parametrize("value", [NAN, INF])
def test_rows_without_an_answer(ctx, classes, value):
    """A NaN or +inf anywhere spoils its row and no other; a given class outside the classes is told."""
    for dtype in (F16, F32):
        x, given = logits(6, classes, dtype, 3)
        x[1, 0] = value
        x[2, classes - 1] = value
        x[3, classes // 3] = value
        x[3, 1] = -INF
        given[2] = -1
        given[4] = classes
        given[5] = 2 ** 31 - 1
        check(ctx, x, given, 5)


@pytest.mark.parametrize("classes", [64, 1000, 4097, 70001])
@pytest.mark.parametrize("order", ["constant", "rising", "falling", "few values", "one block", "every 64th", "every 256th", "signed zeros", "peak", "tiny"])
def test_orders_and_ties(ctx, classes, order):
    i = torch.arange(classes)
    x = {"constant": torch.full((classes,), -3.5), "rising": i * 1e-3, "falling": -i * 1e-3, "few values": (i * 7919 % 5).float(),
         "one block": torch.where((i > classes // 2) & (i < classes // 2 + 400), 5.0 + (i % 17) * 0.1, (i % 29) * 0.01),
         "every 64th": torch.where(i % 64 == 5, 4.0 + (i * 31 % 101) * 0.01, 0.0), "every 256th": torch.where(i % 256 == 255, 3.0, -(i % 3).float()),
         "signed zeros": torch.where(i % 2 == 0, -0.0, 0.0), "peak": torch.where(i == classes - 1, 90.0, 0.0),
         "tiny": (i * 7919 % 1009) * 1e-40}[order].float()
    for dtype in (F32, F16):
        for top in (1, 20, 64):
            check(ctx, x.to(dtype)[None].repeat(2, 1), torch.tensor([classes // 2, classes - 1], dtype=torch.int32), top, what=(dtype, top))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("gap", [1, 3, 8])
def test_strides(ctx, dtype, gap):
    """Rows that are parts of wider ones, from odd addresses on, with NaN around them; one row for all; rows 2^32 bytes apart."""
    for rows, classes in ((3, 1001), (2, 50000)):
        x, given = logits(rows, classes, dtype, gap)
        ref = answer_ref(x, given, 7, 1.0)
        wide = torch.full((rows + 2, classes + 2 * gap), NAN, dtype=dtype, device="cuda")
        part = wide[1:-1, gap:gap + classes]
        part.copy_(x)
        for ws in (None, new_workspace(ctx)):
            assert_answer({k: v.cpu() for k, v in call(ctx, part, given.cuda(), 7, workspace=ws).items()}, ref)
            one = call(ctx, part[:1].expand(rows, -1), given[:1].cuda().repeat(rows), 7, workspace=ws)
            assert all(torch.equal(v, v[:1].expand_as(v)) for v in one.values())


def test_rows_far_apart(ctx):
    x, given = logits(2, 3000, F16, 4)
    store = torch.empty((1 << 31) + (1 << 16), dtype=F16, device="cuda")
    far_apart = store.as_strided((2, 3000), ((1 << 31) + 8, 1))
    far_apart.copy_(x)
    assert_answer({k: v.cpu() for k, v in call(ctx, far_apart, given.cuda(), 4).items()}, answer_ref(x, given, 4, 1.0))


def test_outputs_that_were_not_asked_for(ctx):
    x, given = logits(4, 2000, F32, 2)
    ref = answer_ref(x, given, 6, 1.0)
    xd, gd, s = x.cuda(), given.cuda(), torch.cuda.current_stream()
    for names in (("logp",), ("rank",), ("entropy",), ("top_id", "top_logp"), ("entropy", "top_id", "top_logp"), ()):
        out = {k: v for k, v in outputs(4, 6).items() if k in names}
        ctx.answer(xd, gd if set(names) & {"logp", "rank"} else None, stream=s, **out)
        assert_answer({k: v.cpu() for k, v in out.items()}, ref)
    ctx.answer(torch.zeros(0, 2000, device="cuda"), None, entropy=torch.zeros(0, device="cuda"), stream=s)


def test_what_lies_behind_the_answers_stays(ctx):
    x, given = logits(3, 500, F16, 2)
    big = {k: torch.full((64,), -9, dtype=torch.int32 if k in ("rank", "top_id") else F32, device="cuda") for k in ("logp", "rank", "entropy", "top_id", "top_logp")}
    out = {k: v[8:11] if k not in ("top_id", "top_logp") else v[8:8 + 12].view(3, 4) for k, v in big.items()}
    call(ctx, x.cuda(), given.cuda(), 4, out=out)
    assert_answer({k: v.cpu() for k, v in out.items()}, answer_ref(x, given, 4, 1.0))
    for k, v in big.items():
        n = 12 if k in ("top_id", "top_logp") else 3
        assert bool((v[:8] == -9).all()) and bool((v[8 + n:] == -9).all())


@pytest.mark.parametrize("rows, classes", [(1, 131072), (16, 1000), (40, 30001), (300, 700)])
def test_same_bits_every_time_on_two_streams_at_once_and_replayed(ctx, rows, classes):
    x, given = logits(rows, classes, BF16, 5)
    x, given = x.cuda(), given.cuda()
    spaces = [new_workspace(ctx) for _ in range(3)]
    want = call(ctx, x, given, 10, workspace=spaces[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [outputs(rows, 10) for _ in range(8)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        call(ctx, x, given, 10, workspace=spaces[i % 2], out=o, stream=streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o[k], want[k]) for o in outs for k in want)
    graphs, out = [torch.cuda.CUDAGraph() for _ in range(2)], outputs(rows, 10)
    for g in graphs:                      # two graphs of one workspace, replayed one behind the other
        with torch.cuda.graph(g):
            call(ctx, x, given, 10, workspace=spaces[2], out=out)
    for i in range(4):
        x.copy_(x.roll(1 + i, 1))
        want = call(ctx, x, given, 10, workspace=spaces[0])
        torch.cuda.synchronize()
        for v in out.values():
            v.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in want)


# Many short rows: of a wave each.
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rows, classes, top", [(513, 1, 1), (600, 37, 5), (520, 64, 64), (515, 1023, 17), (514, 2047, 64), (513, 2048, 20), (530, 2049, 9)])
def test_many_short_rows(ctx, rows, classes, top, dtype):
    x, given = logits(rows, classes, dtype, seed=rows + classes)
    x[5] = x[5, 0]                                     # ties everywhere
    x[6] = (x[6].float() * 0.3).round().to(dtype)      # and many
    x[7] = -INF
    x[8, 1:] = -INF
    x[9, classes // 2] = NAN
    x[10, classes // 3] = INF
    x[11, ::2] = torch.finfo(dtype).min
    x[12] = x[12].sort().values
    given[13:17] = torch.tensor([-1, classes, classes - 1, 0], dtype=torch.int32)
    check(ctx, x, given, top, 0.9)


@pytest.mark.parametrize("rows, classes", [(2, 300), (3, 20011)])
@pytest.mark.parametrize("scale", [1e-38, 3.4e38])
def test_scales_near_the_ends_of_the_range(ctx, rows, classes, scale):
    x = torch.full((rows, classes), -2.0)
    x[:, 7:classes:40] = 1.5
    check(ctx, x, torch.full((rows,), 47, dtype=torch.int32), 5, scale)


@pytest.mark.parametrize("classes", [1 << 17, (1 << 20) + 77, 1 << 24])
@pytest.mark.parametrize("order", ["one above the rest", "few values", "rising", "rising fast", "random"])
def test_sums_of_many_classes_keep_their_bits(ctx, classes, order):
    """Rows that one workgroup walks, whose terms are alike and round alike.  In units of 2^-24 (mean and square: of |d| and d^2 under the probabilities): S of 32
    terms in a row, then in more bits, then of 64 lanes and 4 waves: 31 + 10; its exponentials 4 + 2 mean; a maximum's rise a few: less than 64 + 8 mean together.
    sum(d e) / S: 31 + 10 + 4 and S's own, each times mean, and 2 square from its exponentials: less than 128 mean + 8 square.  The last logarithm, product and
    difference: two steps of what they give."""
    i = torch.arange(classes, device="cuda")
    x = {"one above the rest": torch.where(i == classes // 3, 0.0, -0.7), "few values": (i * 7919 % 5) * -0.3, "rising": i * (1.0 / (1 << 24)),
         "rising fast": i * (20.0 / classes), "random": torch.randn(classes, device="cuda", generator=torch.Generator("cuda").manual_seed(3)) * 2.5}[order].float()[None]
    given = torch.tensor([classes // 3], dtype=torch.int32, device="cuda")
    got = {k: v[0].tolist() for k, v in call(ctx, x, given, 3).items()}
    d = x[0].double() - x[0].double().max()
    e = d.exp()
    s = float(e.sum())
    ls, mean, square = math.log(s), float(-(d * e).sum()) / s, float((d * d * e).sum()) / s
    far = 2.0 ** -24 * (64 + 8 * mean)
    step = 2.0 ** -22
    for have, at in [(got["logp"], classes // 3)] + list(zip(got["top_logp"], got["top_id"])):
        assert abs(have - (float(d[at]) - ls)) <= far + step * (abs(float(d[at])) + ls)
    assert abs(got["entropy"] - (ls + mean)) <= 2.0 ** -24 * (64 + 128 * mean + 8 * square) + step * (ls + mean)
    assert got["rank"] == int(((x[0] > x[0, classes // 3]) | ((x[0] == x[0, classes // 3]) & (i < classes // 3))).sum())


@pytest.mark.parametrize("rows, cin, classes, x, z", [(1, 512, 1000, F32, F32), (5, 1024, 20011, F16, F16), (64, 640, 3001, BF16, F32)])
def test_from_features_to_the_answer(ctx, rows, cin, classes, x, z):
    """The end of a network as it is used: 4-bit layer, then the answer over its logits, on one stream and as one graph."""
    d = fc4_data(rows, cin, classes, 64, x, F16, True, seed=13)
    g = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in d.items()}
    given = (torch.arange(rows, dtype=torch.int32) * 37 % classes).cuda()
    y, out, workspace = torch.zeros(rows, classes, dtype=z, device="cuda"), outputs(rows, 8), new_workspace(ctx)

    def both():
        s = torch.cuda.current_stream()
        ctx.fc4(g["x"], g["q"], g["scales"], y, 64, zeros=g["zeros"], bias=g["bias"], stream=s)
        ctx.answer(y, given, scale=0.8, workspace=workspace, stream=s, **out)

    def right():
        assert_fc4(y.cpu(), *fc4_ref(d))
        assert_answer({k: v.cpu() for k, v in out.items()}, answer_ref(y.cpu(), given.cpu(), 8, 0.8))

    both()
    torch.cuda.synchronize()
    right()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        d["x"] = d["x"].roll(1, 1)
        g["x"].copy_(d["x"])
        graph.replay()
        torch.cuda.synchronize()
        right()
