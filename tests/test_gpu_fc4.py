"""cw_fc4 against 64 bits: sizes from one on, types, strides, special values, streams and graphs, and CW_OP_FC4 inside a model."""
import pytest
import torch

import paper_2006_02464_amd as cw
from operator_refs import assert_fc4, fc4_data, fc4_ref, fc4_weights

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = cw.Context(workspace_bytes=16 << 20, io_bytes=1 << 20, weight_pool_bytes=16 << 20, load_staging_bytes=1 << 20)
    yield c
    c.destroy()


def on_gpu(d):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in d.items()}


def call(ctx, d, y, bias=True, stream=None):
    ctx.fc4(d["x"], d["q"], d["scales"], y, d["group"], zeros=d["zeros"], bias=d["bias"] if bias else None,
            stream=torch.cuda.current_stream() if stream is None else stream)


def check(ctx, rows, cin, cout, group, x=F16, scale=F16, y=F32, zeros=False, seed=0, spread=False):
    d = fc4_data(rows, cin, cout, group, x, scale, zeros, seed, spread)
    out = torch.full((rows, cout), float("nan"), dtype=y, device="cuda")
    call(ctx, on_gpu(d), out)
    assert_fc4(out.cpu(), *fc4_ref(d))


SIZES = [(1, 1, 1, 32), (1, 2, 3, 32), (2, 5, 16, 32), (3, 31, 17, 32), (1, 32, 1, 32), (1, 33, 15, 32), (4, 63, 64, 64), (7, 64, 65, 64), (8, 65, 5, 64),
         (15, 127, 33, 128), (16, 128, 130, 128), (17, 129, 48, 128), (1, 200, 777, 32), (5, 1000, 777, 32), (31, 96, 100, 96), (33, 500, 129, 96),
         (1, 2048, 1000, 128), (16, 512, 1000, 64), (1, 4097, 40, 128), (2, 6144, 33, 256), (32, 640, 72, 512), (64, 1024, 200, 64), (65, 256, 90, 32),
         (100, 320, 256, 32), (128, 512, 128, 64), (129, 384, 257, 128), (257, 288, 66, 96), (300, 1027, 131, 32), (512, 64, 16, 64), (1, 16384, 20, 1024),
         (9, 8192, 24, 8192), (48, 2500, 50, 64)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("types", [(F16, F16, F16, False), (BF16, BF16, F32, True), (F32, F16, F32, True)], ids=["fp16", "bf16", "fp32"])
def test_sizes(ctx, size, types):
    x, scale, y, zeros = types
    check(ctx, *size, x=x, scale=scale, y=y, zeros=zeros, seed=sum(size))


# Wide enough for the forms that share activations between many weight rows or walk over tiles, with rows that end inside a block, and long enough that
# the scales come in several lots.
WIDE = [(1, 160, 16500, 32), (5, 200, 16433, 96), (16, 2200, 12900, 64), (16, 4000, 500, 32), (13, 10016, 40, 32), (24, 200, 12900, 64), (500, 300, 850, 128), (500, 168, 1700, 32),
        (500, 264, 3300, 64), (450, 5000, 3300, 32), (30, 12000, 50, 32), (40, 3840, 33, 480)]


@pytest.mark.parametrize("size", WIDE, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("types", [(F16, F16, F32, True), (BF16, BF16, F32, False), (BF16, F16, BF16, True), (F32, F32, F32, True)], ids=["fp16", "bf16", "bf16 plain", "fp32"])
def test_wide_and_long(ctx, size, types):
    x, scale, y, zeros = types
    check(ctx, *size, x=x, scale=scale, y=y, zeros=zeros, seed=sum(size))


# A size for each tile of the forms for many rows, from 16 x 16 to 128 x 256 (the largest is 64 x 256 for what takes more registers).
TILES = [(13, 10016, 40), (16, 2600, 4200), (16, 2600, 8300), (200, 420, 1000), (24, 200, 8500), (40, 420, 9000), (100, 420, 9000), (500, 420, 4100), (1000, 290, 4100)]


@pytest.mark.parametrize("size", TILES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("types", [(F16, F16), (BF16, F32), (BF16, BF16), (F32, F32)], ids=["fp16", "bf16", "bf16 plain", "fp32"])
def test_every_tile(ctx, size, group, zeros, types):
    check(ctx, *size, group, types[0], BF16, types[1], zeros, seed=group)


@pytest.mark.parametrize("rows, group, zeros", [(1, 32, True), (2, 64, False), (2, 96, True), (1, 128, False), (3, 128, True)])
@pytest.mark.parametrize("x", [F16, BF16, F32])
def test_long_rows_to_a_large_vocabulary(ctx, rows, group, zeros, x):
    check(ctx, rows, 4100, 16410, group, x, F16, x, zeros, seed=rows + group)


@pytest.mark.parametrize("x", [F16, BF16, F32])
@pytest.mark.parametrize("scale", [F16, BF16, F32])
@pytest.mark.parametrize("y", [F16, BF16, F32])
def test_types(ctx, x, scale, y):
    for zeros in (False, True):
        check(ctx, 6, 328, 70, 64, x, scale, y, zeros, seed=3)
        check(ctx, 70, 328, 70, 64, x, scale, y, zeros, seed=4)


@pytest.mark.parametrize("x", [BF16, F32])
@pytest.mark.parametrize("size", [(3, 700, 40, 32), (90, 1400, 40, 128)])
def test_activations_of_many_magnitudes(ctx, x, size):
    check(ctx, *size, x=x, scale=F32, y=F32, seed=11, spread=True)


@pytest.mark.parametrize("x, y, power", [(BF16, BF16, 112), (BF16, F32, 120), (F32, F32, 120), (BF16, BF16, -110), (F32, F32, -110)])
@pytest.mark.parametrize("rows", [3, 70])
def test_activations_near_the_ends_of_the_range(ctx, x, y, power, rows):
    d = fc4_data(rows, 392, 40, 64, x, F32, True, seed=12)
    d["x"] = d["x"] * 2.0 ** power
    d["bias"] = d["bias"] * 2.0 ** power
    out = torch.full((rows, 40), float("nan"), dtype=y, device="cuda")
    call(ctx, on_gpu(d), out)
    assert_fc4(out.cpu(), *fc4_ref(d))


@pytest.mark.parametrize("x", [F16, BF16, F32])
@pytest.mark.parametrize("rows", [1, 5, 20, 130])
@pytest.mark.parametrize("gap", [1, 8, 16])
def test_strides_and_what_lies_between_the_rows(ctx, x, rows, gap):
    """Every tensor a part of a wider one, beginning `gap` elements in: odd addresses and strides; what is not y's stays as it was."""
    cin, cout, group = 264, 75, 64
    d = on_gpu(fc4_data(rows, cin, cout, group, x, F16, True, seed=gap))

    def inside(t, fill):
        wide = torch.full((t.shape[0] + 2, t.shape[1] + 2 * gap), fill, dtype=t.dtype, device="cuda")
        part = wide[1:-1, gap:gap + t.shape[1]]
        part.copy_(t)
        return part

    s = dict(d, **{k: inside(d[k], 255 if d[k].dtype == torch.uint8 else float("nan")) for k in ("x", "q", "scales", "zeros")})
    wide = torch.full((rows + 2, cout + 2 * gap), 7.0, device="cuda", dtype=F32)
    call(ctx, s, wide[1:-1, gap:gap + cout])
    assert_fc4(wide[1:-1, gap:gap + cout].cpu(), *fc4_ref({k: v.cpu() if isinstance(v, torch.Tensor) else v for k, v in d.items()}))
    keep = torch.ones_like(wide, dtype=torch.bool)
    keep[1:-1, gap:gap + cout] = False
    assert bool((wide[keep] == 7.0).all())


def test_one_row_for_all_and_one_weight_row_for_all(ctx):
    d = fc4_data(1, 200, 50, 32, F16, F16, True, seed=2)
    y, far = fc4_ref(d)
    g = on_gpu(d)
    for rows in (3, 40, 200):
        out = torch.zeros(rows, 50, device="cuda")
        call(ctx, dict(g, x=g["x"].expand(rows, -1)), out)
        assert_fc4(out.cpu(), y.expand(rows, -1), far.expand(rows, -1))
        one = {k: g[k][:1].expand(50, -1) for k in ("q", "scales", "zeros")}
        call(ctx, dict(g, x=g["x"].expand(rows, -1), **one), out, bias=False)
        assert bool((out == out[0, 0]).all())


@pytest.mark.parametrize("big", ["x", "q", "scales", "zeros", "y"])
def test_offsets_beyond_32_bits(ctx, big):
    """Rows that lie more than 2^31 bytes (and elements, of bytes) apart."""
    rows, cin, cout = 3, 160, 3
    d = on_gpu(fc4_data(rows, cin, cout, 32, F16, F16, True, seed=9))
    out = torch.zeros(rows, cout, device="cuda", dtype=F16)
    stride = (1 << 31) + 64 if big in ("q", "zeros") else (1 << 30) + 32
    src = out if big == "y" else d[big]
    store = torch.empty(2 * stride + 4096, dtype=src.dtype, device="cuda")
    far_apart = store.as_strided(src.shape, (stride, 1))
    far_apart.copy_(src)
    if big == "y":
        out = far_apart
    else:
        d[big] = far_apart
    call(ctx, d, out)
    assert_fc4(out.cpu(), *fc4_ref({k: v.cpu() if isinstance(v, torch.Tensor) else v for k, v in d.items()}))


@pytest.mark.parametrize("x", [F16, BF16, F32])
@pytest.mark.parametrize("rows", [4, 100])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_a_special_activation_stays_in_its_row(ctx, x, rows, value):
    d = fc4_data(rows, 300, 40, 32, x, F16, True, seed=5)
    y, far = fc4_ref(d)
    d["x"][2, 37] = value
    out = torch.zeros(rows, 40, device="cuda")
    call(ctx, on_gpu(d), out)
    out = out.cpu()
    others = torch.arange(rows) != 2
    assert not torch.isfinite(out[2]).any()
    assert_fc4(out[others], y[others], far[others])


@pytest.mark.parametrize("rows", [4, 100])
def test_a_special_scale_stays_in_its_column(ctx, rows):
    d = fc4_data(rows, 300, 40, 32, F16, F16, True, seed=6)
    y, far = fc4_ref(d)
    d["scales"][7, 9] = float("nan")
    d["scales"][8, 0] = 0.0
    d["zeros"] |= 0xA0                       # only the low four bits count
    out = torch.zeros(rows, 40, device="cuda")
    call(ctx, on_gpu(d), out)
    out = out.cpu()
    assert torch.isnan(out[:, 7]).all()
    same = [n for n in range(40) if n not in (7, 8)]
    assert_fc4(out[:, same], y[:, same], far[:, same])
    d["zeros"] &= 15
    d["scales"][7, 9] = 0.0
    y, far = fc4_ref(d)
    assert_fc4(out[:, 8:9], y[:, 8:9], far[:, 8:9])


def test_zeros_and_largest_values(ctx):
    """Rows of zeros, activations of the type's largest magnitude, subnormal scales."""
    for x, most in ((F16, 65504.0), (BF16, 2.0 ** 100), (F32, 2.0 ** 100)):
        d = fc4_data(20, 160, 30, 32, x, F32, True, seed=8)
        d["x"][3] = 0
        d["x"][5] = most
        d["x"][6] = 2.0 ** -20
        d["x"][7, ::2] = 0
        d["scales"][4] = 2.0 ** -130
        d["bias"][4] = 0
        out = torch.full((20, 30), 1.0, device="cuda")
        call(ctx, on_gpu(d), out)
        y, far = fc4_ref(d)
        assert torch.equal(out[3].cpu(), d["bias"])
        at = [n for n in range(30) if n != 4]
        assert_fc4(out.cpu()[:, at], y[:, at], far[:, at])
        # products of a subnormal scale: their own roundings are steps of 2^-149
        off = (out[:, 4].cpu().double() - y[:, 4]).abs()
        assert bool((off <= far[:, 4] + 160 * 2.0 ** -149 * d["x"].double().abs().amax(1).clamp(min=1)).all())


def test_no_bias_no_rows(ctx):
    d = fc4_data(3, 100, 20, 32, F16, F16, seed=1)
    d["bias"].zero_()
    out = torch.zeros(3, 20, device="cuda")
    call(ctx, on_gpu(d), out, bias=False)
    assert_fc4(out.cpu(), *fc4_ref(d))
    none = dict(on_gpu(d), x=torch.zeros(0, 100, device="cuda", dtype=F16))
    call(ctx, none, torch.zeros(0, 20, device="cuda"))


@pytest.mark.parametrize("size", [(1, 700, 333, 64), (20, 700, 333, 64), (200, 700, 333, 64)])
def test_same_bits_every_time_on_two_streams_at_once_and_replayed(ctx, size):
    d = on_gpu(fc4_data(*size, BF16, BF16, True, seed=7))
    want = torch.zeros(size[0], size[2], device="cuda")
    call(ctx, d, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(want) for _ in range(8)]
    for i, o in enumerate(outs):
        call(ctx, d, o, stream=streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(want)
    with torch.cuda.graph(graph):
        call(ctx, d, out)
    for i in range(3):
        d["x"].mul_(-1.0)
        call(ctx, d, want)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def at_the_zero_point(d, channels):
    """The weights of these inputs become zero: nibble = zero point."""
    d["nib"][:, channels] = d["zeros"][:, channels // d["group"]] if d["zeros"] is not None else 8
    wide = torch.zeros(d["nib"].shape[0], d["q"].shape[1] * 2, dtype=torch.uint8)
    wide[:, :d["nib"].shape[1]] = d["nib"]
    d["q"] = wide[:, 0::2] | (wide[:, 1::2] << 4)


@pytest.mark.parametrize("rows", [5, 70, 500])
@pytest.mark.parametrize("group, zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("x, loud", [(F16, 3000.0), (BF16, 3e4), (F32, 3e4)], ids=["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("y", [F16, BF16, F32], ids=["to fp16", "to bf16", "to fp32"])
def test_a_loud_activation_at_the_zero_point_takes_nothing_from_the_others(ctx, rows, group, zeros, x, loud, y):
    """One input in every 128 is thousands of times the others, and all of its weights are zero."""
    d = fc4_data(rows, 520, 300, group, x, F16, zeros, seed=14)
    channels = torch.arange(5, 520, 128)
    d["x"][:, channels] *= loud
    at_the_zero_point(d, channels)
    out = torch.full((rows, 300), float("nan"), dtype=y, device="cuda")
    call(ctx, on_gpu(d), out)
    assert_fc4(out.cpu(), *fc4_ref(d))


@pytest.mark.parametrize("x", [F16, BF16, F32])
@pytest.mark.parametrize("y", [F16, BF16, F32])
@pytest.mark.parametrize("rows, cin", [(5, 20), (5, 300), (100, 300), (100, 411)])
def test_infinities_come_out_as_the_definition_has_them(ctx, x, y, rows, cin):
    """x (q - z) s of an infinite x: an infinity of the product's sign, no number where the weight is zero or infinities of both signs meet."""
    d = fc4_data(rows, cin, 40, 32, x, F16, True, seed=15)
    inf = float("inf")
    d["x"][0, 7] = inf
    d["x"][1, cin - 1] = -inf
    d["x"][2, 3], d["x"][2, 17] = inf, -inf
    d["x"][3, 0], d["x"][3, 11] = -inf, float("nan")
    d["x"][rows - 1, 2:9:3] = -inf
    d["scales"][6] = 0.0
    out = torch.zeros(rows, 40, dtype=y, device="cuda")
    call(ctx, on_gpu(d), out)
    out = out.cpu()
    special = [0, 1, 2, 3, rows - 1]
    want = (d["x"][special].double()[:, None] * fc4_weights(d)).sum(2)
    assert not torch.isfinite(want).any() and torch.isinf(want).any() and torch.isnan(want).any()
    assert torch.equal(out[special].double().nan_to_num(7.0, inf, -inf), want.nan_to_num(7.0, inf, -inf))
    d["x"][special] = 0.0
    others = [m for m in range(rows) if m not in special]
    assert_fc4(out[others], *(v[others] for v in fc4_ref(d)))


@pytest.mark.parametrize("rows", [16, 100])
@pytest.mark.parametrize("x, most", [(F16, 1.0), (F16, 1.9921875)] + [(x, most) for x in (BF16, F32) for most in (1.0, 1.9921875, 2.0 ** 100, 1.5 * 2.0 ** -100)])
def test_what_is_kept_of_an_activation_beside_a_larger_one(ctx, rows, x, most):
    """Each row has one input of weight 0, the largest, and one of weight 1, smaller by more from row to row: the result is what stands for it, no sum and no
    rounding of its own.  The bounds are the header's."""
    g = torch.Generator().manual_seed(18)
    d = fc4_data(rows, 130, 16, 128, x, F32, False, seed=18)
    d["x"].zero_()
    d["x"][:, 40] = most
    small = ((1.0 + torch.rand(rows, generator=g)) * 0.5 * most * 2.0 ** -(torch.arange(rows) % 48).double()).to(x)
    d["x"][:, 77] = small * (1 - 2 * (torch.arange(rows) % 2)).to(x)
    d["nib"][:, 77] = 9
    at_the_zero_point(d, torch.tensor([40]))
    d["scales"].fill_(1.0)
    d["bias"].zero_()
    out = torch.full((rows, 16), float("nan"), device="cuda")
    call(ctx, on_gpu(d), out)
    have, want = out.cpu().double(), d["x"][:, 77:78].double()
    off = (have - want).abs()
    if x == F16:
        assert bool((off == 0).all())
    elif x == BF16:
        assert bool((off < 2.0 ** -38 * most).all()) and bool((off[want[:, 0].abs() >= 2.0 ** -31 * most] == 0).all())
    else:
        assert bool((off <= 2.0 ** -23 * want.abs() + 2.0 ** -39 * most).all())


@pytest.mark.parametrize("group", [1 << 20, 1 << 30, (1 << 31) - 64, (1 << 31) - 32])
@pytest.mark.parametrize("rows, cin", [(1, 20), (3, 4096), (16, 1000), (40, 4096), (130, 1000)])
def test_a_group_longer_than_the_rows(ctx, group, rows, cin):
    for zeros in (False, True):
        check(ctx, rows, cin, 50, group, F16, F16, F32, zeros, seed=16)
        check(ctx, rows, cin, 50, group, F32, F32, F32, zeros, seed=17)


# ---- as an operator of a model ---------------------------------------------------------------------
def fc4_model(dtype, classes, group):
    """A small network with FC4 in the place of FC, its blob, and the same network with the weights that the 4 bits stand for."""
    import numpy as np

    from oracle import topology as T
    from workload import gen
    plain = [T.Op(T.CONV, 3, 64, 3, 3, 2, 1, 1, -1, -1), T.Op(T.CONV, 64, 320, 1, 1, 1, 0, 1, -1, 0), T.Op(T.GAVGPOOL, 320, 320, 0, 0, 1, 0, 0, -1, 1),
             T.Op(T.FC, 320, classes, 1, 1, 1, 0, 0, -1, 2), T.Op(T.SOFTMAX, classes, classes, 0, 0, 1, 0, 0, -1, 3)]
    ops = list(map(tuple, plain))
    ops[3] = (cw.CW_OP_FC4, 320, classes, 1, 1, 1, 0, 0, -1, 2, 0, group)
    w, b = gen.model_tensors(T.weight_shapes(plain), 5, dtype)
    d = fc4_data(1, 320, classes, group, F32, F16 if dtype == "fp16" else BF16, True, seed=21)
    raw = lambda t: t.contiguous().view(torch.uint8).numpy().tobytes()
    even = lambda s: s + b"\0" * (len(s) % 2)
    half = lambda a: raw(torch.from_numpy(np.ascontiguousarray(a)).to(F16 if dtype == "fp16" else BF16))
    weights = half(w[0]) + half(w[1]) + even(raw(d["q"])) + even(raw(d["scales"])) + even(raw(d["zeros"]))
    weights += b"\0" * (-len(weights) % 4)
    blob = np.frombuffer(weights + b"".join(np.ascontiguousarray(v, np.float32).tobytes() for v in b), np.uint8)
    w[2] = fc4_weights(d).float().numpy().reshape(w[2].shape)
    return ops, blob, plain, w, b


@pytest.mark.parametrize("dtype, classes, group", [("fp16", 1000, 64), ("bf16", 33, 96), ("fp16", 7, 32)])
def test_fc4_in_a_model(dtype, classes, group):
    """LOAD, EXEC in both forms, OUTPUT of the rows and of the answer, against the oracle over the weights that the 4 bits stand for."""
    import numpy as np

    from gpu_common import TOL, rel_err_per_sample
    from operator_refs import answer_ref, assert_answer
    from oracle import network as N
    from paper_2006_02464_amd.runner import Worker, pinned_like
    from workload import gen
    ops, blob, plain, w, b = fc4_model(dtype, classes, group)
    wk = Worker(workspace_bytes=64 << 20, io_bytes=8 << 20, weight_pool_bytes=64 << 20, load_staging_bytes=8 << 20)
    try:
        ctx = wk.ctx
        mid = ctx.model_define(ops, 3, 30, 30, batch_sizes=(1, 3, 16), dtype=dtype)
        assert ctx.model_weight_bytes(mid) == blob.size
        wk.load(mid, blob)
        x = gen.images(5, 0, 16, 3, 30, 30, "normal", dtype)
        want = N.forward(plain, w, b, x, prec="f32", keep="final", storage=None)["logits"]
        for batch in (16, 3, 1):
            xs = x[:batch]
            probs, logits, _ = wk.infer(mid, xs, classes)
            assert rel_err_per_sample(logits, want[:batch]).max() <= TOL
            xd, z, p = torch.from_numpy(np.ascontiguousarray(xs)).cuda(), torch.zeros(batch, classes, device="cuda"), torch.zeros(batch, classes, device="cuda")
            torch.cuda.synchronize()
            ctx.exec_static(mid, batch, xd, z, p, wk.stream)
            wk.stream.synchronize()
            assert np.array_equal(z.cpu().numpy(), logits) and np.array_equal(p.cpu().numpy(), probs)
            hx, given = pinned_like(np.ascontiguousarray(xs, dtype=np.float32)), pinned_like(np.arange(batch, dtype=np.int32) % classes)
            for pinned in (True, False):
                top = min(5, classes)
                host = torch.full((ctx.answer_bytes(batch, top) + 16,), 85, dtype=torch.uint8)
                host = host.pin_memory() if pinned else host
                slot = ctx.input(mid, batch, hx, wk.stream)
                ctx.exec(mid, batch, slot, wk.stream)
                ctx.output_answer(slot, host, given, top, 0.5, wk.stream)
                wk.stream.synchronize()
                assert bool((host[-16:] == 85).all())
                got = {k: torch.from_numpy(v.copy()) for k, v in ctx.split_answer(host, batch, top).items()}
                assert_answer(got, answer_ref(torch.from_numpy(logits), given, top, 0.5))
                with pytest.raises(cw.CwError) as e:       # the slot is released
                    ctx.output_answer(slot, host, given, top, 0.5, wk.stream)
                assert e.value.status == cw.CW_ERR_NO_INPUT
        ctx.unload_weights(mid)
        wk.load(mid, blob)
        again = wk.infer(mid, x, classes)[1]
        assert rel_err_per_sample(again, want).max() <= TOL
    finally:
        wk.close()


def test_output_answer_refuses_arrays_of_other_sizes():
    """Too few given classes, or too many, and too little room: nothing is read or written, and the slot stays."""
    import numpy as np

    from operator_refs import answer_ref, assert_answer
    from paper_2006_02464_amd.runner import Worker, pinned_like
    from workload import gen
    ops, blob, _, _, _ = fc4_model("fp16", 33, 64)
    wk = Worker(workspace_bytes=64 << 20, io_bytes=8 << 20, weight_pool_bytes=64 << 20, load_staging_bytes=8 << 20)
    try:
        ctx = wk.ctx
        mid = ctx.model_define(ops, 3, 30, 30, batch_sizes=(3,), dtype="fp16")
        wk.load(mid, blob)
        x = gen.images(5, 0, 3, 3, 30, 30, "normal", "fp16")
        logits = torch.from_numpy(wk.infer(mid, x, 33)[1])
        slot = ctx.input(mid, 3, pinned_like(np.ascontiguousarray(x, dtype=np.float32)), wk.stream)
        assert ctx.slot_batch(slot) == 3
        ctx.exec(mid, 3, slot, wk.stream)
        given, host = torch.tensor([5, 0, 32], dtype=torch.int32), torch.zeros(ctx.answer_bytes(3, 4), dtype=torch.uint8)
        for change in (dict(given=given[:2]), dict(given=given.repeat(2)), dict(given=given.long()), dict(given=given.cuda()), dict(host_answer=host[:-1]), dict(host_answer=host.cuda())):
            with pytest.raises(ValueError):
                ctx.output_answer(**dict(dict(slot=slot, host_answer=host, given=given, top=4, stream=wk.stream), **change))
        assert ctx.slot_batch(slot) == 3 and not bool(host.any())
        ctx.output_answer(slot, host, given, 4, stream=wk.stream)
        wk.stream.synchronize()
        assert_answer({k: torch.from_numpy(v.copy()) for k, v in ctx.split_answer(host, 3, 4).items()}, answer_ref(logits, given, 4, 1.0))
    finally:
        wk.close()
