"""What cw_fc4, cw_answer and cw_output_answer refuse, on a planning-only context: every check stands before the first use of the GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2006_02464_amd as cw
from oracle import topology as T


@pytest.fixture()
def ctx():
    c = cw.Context(device=-1)
    yield c
    c.destroy()


def fc4_args(**change):
    a = dict(x=4096, q=4096, scales=4096, zeros=4096, bias=4096, y=4096, x_stride=100, q_stride=50, scale_stride=4, zero_stride=4, y_stride=20, rows=3, cin=100, cout=20, group=32,
             x_dtype=0, scale_dtype=0, y_dtype=2)
    a.update(change)
    return cw.cw_fc4_args(*[a[n] for n, _ in cw.cw_fc4_args._fields_])


def answer_args(**change):
    a = dict(logits=4096, given=4096, logp=4096, rank=4096, entropy=4096, top_id=4096, top_logp=4096, workspace=4096, workspace_bytes=1 << 20, stride=50, rows=3, classes=50,
             top=5, dtype=2, scale=1.0)
    a.update(change)
    return cw.cw_answer_args(*[a[n] for n, _ in cw.cw_answer_args._fields_])


def refusal(ctx, call, args):
    st = call(ctx._h, ctypes.byref(args), None)
    return st, cw.lib().cw_last_error(ctx._h).decode()


PLANNING = (cw.CW_ERR_INVALID, "planning-only context has no device")


@pytest.mark.parametrize("change, status", [
    (dict(x=None), cw.CW_ERR_INVALID), (dict(q=None), cw.CW_ERR_INVALID), (dict(scales=None), cw.CW_ERR_INVALID), (dict(y=None), cw.CW_ERR_INVALID),
    (dict(x=4097), cw.CW_ERR_INVALID), (dict(x=4098, x_dtype=2), cw.CW_ERR_INVALID), (dict(scales=4097), cw.CW_ERR_INVALID), (dict(y=4098), cw.CW_ERR_INVALID),
    (dict(bias=4098), cw.CW_ERR_INVALID), (dict(rows=-1), cw.CW_ERR_INVALID), (dict(cin=0), cw.CW_ERR_INVALID), (dict(cout=0), cw.CW_ERR_INVALID),
    (dict(cin=(1 << 24) + 1), cw.CW_ERR_UNSUPPORTED), (dict(rows=(1 << 20) + 1), cw.CW_ERR_UNSUPPORTED), (dict(cout=(1 << 24) + 1), cw.CW_ERR_UNSUPPORTED),
    (dict(group=0), cw.CW_ERR_UNSUPPORTED), (dict(group=16), cw.CW_ERR_UNSUPPORTED), (dict(group=48), cw.CW_ERR_UNSUPPORTED), (dict(group=-32), cw.CW_ERR_UNSUPPORTED),
    (dict(x_stride=-1), cw.CW_ERR_INVALID), (dict(q_stride=-1), cw.CW_ERR_INVALID), (dict(scale_stride=-4), cw.CW_ERR_INVALID), (dict(zero_stride=-4), cw.CW_ERR_INVALID),
    (dict(y_stride=19), cw.CW_ERR_INVALID), (dict(x_dtype=3), cw.CW_ERR_INVALID), (dict(scale_dtype=-1), cw.CW_ERR_INVALID), (dict(y_dtype=7), cw.CW_ERR_INVALID)])
def test_fc4_refuses(ctx, change, status):
    st, why = refusal(ctx, cw.lib().cw_fc4, fc4_args(**change))
    assert st == status and (st, why) != PLANNING


@pytest.mark.parametrize("change", [{}, dict(zeros=None, zero_stride=-5), dict(bias=None), dict(q=4097, zeros=4099, x=4098), dict(x_stride=0, q_stride=0, scale_stride=0, zero_stride=0),
                                    dict(rows=1, y_stride=0), dict(rows=0, x=None, y=None, q=None, scales=None), dict(group=1 << 30), dict(cin=1, group=64)])
def test_fc4_checks_let_through(ctx, change):
    assert refusal(ctx, cw.lib().cw_fc4, fc4_args(**change)) == PLANNING


@pytest.mark.parametrize("change, status", [
    (dict(logits=None), cw.CW_ERR_INVALID), (dict(given=None), cw.CW_ERR_INVALID), (dict(given=None, logp=None), cw.CW_ERR_INVALID), (dict(top_id=None), cw.CW_ERR_INVALID),
    (dict(top_logp=None), cw.CW_ERR_INVALID), (dict(top=0), cw.CW_ERR_INVALID), (dict(top=-1), cw.CW_ERR_UNSUPPORTED), (dict(top=65), cw.CW_ERR_UNSUPPORTED),
    (dict(rows=-1), cw.CW_ERR_INVALID), (dict(classes=0), cw.CW_ERR_INVALID), (dict(classes=(1 << 24) + 1), cw.CW_ERR_UNSUPPORTED), (dict(rows=(1 << 23) + 1), cw.CW_ERR_UNSUPPORTED), (dict(dtype=3), cw.CW_ERR_INVALID),
    (dict(scale=0.0), cw.CW_ERR_INVALID), (dict(scale=-1.0), cw.CW_ERR_INVALID), (dict(scale=float("inf")), cw.CW_ERR_INVALID), (dict(scale=float("nan")), cw.CW_ERR_INVALID),
    (dict(stride=-1), cw.CW_ERR_INVALID), (dict(logits=4098), cw.CW_ERR_INVALID), (dict(logits=4097, dtype=0), cw.CW_ERR_INVALID), (dict(given=4098), cw.CW_ERR_INVALID),
    (dict(logp=4098), cw.CW_ERR_INVALID), (dict(rank=4098), cw.CW_ERR_INVALID), (dict(entropy=4098), cw.CW_ERR_INVALID), (dict(top_id=4098), cw.CW_ERR_INVALID),
    (dict(top_logp=4098), cw.CW_ERR_INVALID), (dict(workspace=4104), cw.CW_ERR_INVALID)])
def test_answer_refuses(ctx, change, status):
    st, why = refusal(ctx, cw.lib().cw_answer, answer_args(**change))
    assert st == status and (st, why) != PLANNING


@pytest.mark.parametrize("change", [{}, dict(workspace=None, workspace_bytes=0), dict(workspace_bytes=8), dict(given=None, logp=None, rank=None), dict(top=0, top_id=None, top_logp=None),
                                    dict(rows=0, logits=None, given=None), dict(stride=0), dict(logits=4098, dtype=1), dict(top=64), dict(classes=1)])
def test_answer_checks_let_through(ctx, change):
    assert refusal(ctx, cw.lib().cw_answer, answer_args(**change)) == PLANNING


def test_null_arguments(ctx):
    for call in (cw.lib().cw_fc4, cw.lib().cw_answer):
        assert call(ctx._h, None, None) == cw.CW_ERR_INVALID
        assert call(None, None, None) == cw.CW_ERR_INVALID
    assert cw.lib().cw_output_answer(None, 0, None, 0, 1.0, None, None) == cw.CW_ERR_INVALID


def test_output_answer_refuses(ctx):
    host = np.zeros(4096, np.uint8)
    for kw, status in ((dict(top=65), cw.CW_ERR_UNSUPPORTED), (dict(top=-1), cw.CW_ERR_UNSUPPORTED), (dict(scale=0.0), cw.CW_ERR_INVALID), ({}, cw.CW_ERR_INVALID)):
        with pytest.raises(cw.CwError) as e:
            ctx.output_answer(0, host, **kw)
        assert e.value.status == status
    with pytest.raises(cw.CwError) as e:
        ctx.output_answer(0, None)
    assert e.value.status == cw.CW_ERR_INVALID


def test_output_answer_refuses_arrays_that_do_not_fit(ctx):
    """Before the call: other types than int32, memory with gaps, memory that cannot be written."""
    host, given = np.zeros(4096, np.uint8), np.zeros(3, np.int32)
    locked = host.copy()
    locked.flags.writeable = False
    for change in (dict(given=given.astype(np.int64)), dict(given=torch.zeros(3, dtype=torch.int64)), dict(given=torch.zeros(3)), dict(given=np.zeros(6, np.int32)[::2]),
                   dict(given=torch.zeros(6, dtype=torch.int32)[::2]), dict(given=given.astype(">i4")), dict(host_answer=host[::2]), dict(host_answer=locked)):
        with pytest.raises(ValueError):
            ctx.output_answer(**dict(dict(slot=0, host_answer=host, given=given), **change))
    with pytest.raises(TypeError):
        ctx.output_answer(0, host, [1, 2, 3])
    for ok in (given, torch.zeros(3, dtype=torch.int32), None):
        with pytest.raises(cw.CwError) as e:
            ctx.output_answer(0, host, ok)
        assert "planning-only" in str(e.value)
    for slot in (-1, 0, 1 << 20):
        with pytest.raises(cw.CwError) as e:
            ctx.slot_batch(slot)
        assert e.value.status == cw.CW_ERR_NO_INPUT


def test_answer_sizes():
    assert cw.Context.answer_bytes(3, 5) == 3 * 52 and cw.Context.answer_bytes(0, 5) == 0 and cw.Context.answer_bytes(7, 0) == 84
    assert cw.Context.answer_bytes(-1, 5) == 0 and cw.Context.answer_bytes(1, 65) == 0 and cw.Context.answer_bytes(1, -1) == 0
    assert cw.CW_ANSWER_COUNTERS <= cw.Context.answer_workspace_bytes() <= 1 << 20
    parts = cw.Context.split_answer(np.arange(3 * 52 + 8, dtype=np.uint8), 3, 5)
    assert {k: v.shape for k, v in parts.items()} == {"logp": (3,), "rank": (3,), "entropy": (3,), "top_id": (3, 5), "top_logp": (3, 5)}


def test_binding_refuses_tensors_that_do_not_fit(ctx):
    """A planning-only context takes CPU tensors: they are on "its" device, -1."""
    x, q, s, y = torch.zeros(3, 100), torch.zeros(20, 50, dtype=torch.uint8), torch.zeros(20, 4), torch.zeros(3, 20)
    ok = dict(x=x, q=q, scales=s, y=y, group=32, zeros=torch.zeros(20, 4, dtype=torch.uint8), bias=torch.zeros(20))
    with pytest.raises(cw.CwError) as e:
        ctx.fc4(**ok)
    assert "planning-only" in str(e.value)
    for change in (dict(q=q[:, :49]), dict(q=q.t().contiguous().t()), dict(scales=s[:, :3]), dict(y=y[:2]), dict(y=torch.zeros(20, 3).t()), dict(zeros=torch.zeros(20, 3, dtype=torch.uint8)),
                   dict(bias=torch.zeros(19)), dict(bias=torch.zeros(40)[::2]), dict(bias=torch.zeros(20, dtype=torch.float16)), dict(group=0)):
        with pytest.raises(ValueError):
            ctx.fc4(**dict(ok, **change))
    for change in (dict(x=x.double()), dict(scales=s.to(torch.int32)), dict(q=q.int()), dict(zeros=torch.zeros(20, 4))):
        with pytest.raises(TypeError):
            ctx.fc4(**dict(ok, **change))
    z, g = torch.zeros(3, 50), torch.zeros(3, dtype=torch.int32)
    f = lambda n=3: torch.zeros(n)
    ok = dict(logits=z, given=g, logp=f(), rank=g.clone(), entropy=f(), top_id=torch.zeros(3, 4, dtype=torch.int32), top_logp=torch.zeros(3, 4), workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(cw.CwError) as e:
        ctx.answer(**ok)
    assert "planning-only" in str(e.value)
    for change in (dict(given=g.long()), dict(given=g[:2]), dict(logp=f(2)), dict(logp=f().double()), dict(rank=f()), dict(entropy=f(4)), dict(top_id=torch.zeros(2, 4, dtype=torch.int32)),
                   dict(top_logp=torch.zeros(3, 5)), dict(logits=torch.zeros(50, 3).t()), dict(workspace=torch.zeros(64))):
        with pytest.raises(ValueError):
            ctx.answer(**dict(ok, **change))
    with pytest.raises(TypeError):
        ctx.answer(**dict(ok, logits=z.double()))


def test_binding_refuses_numbers_out_of_range_as_the_library_does(ctx):
    """A group or a number of rows beyond 32 bits and a scale beyond fp32: the library's error; no numbers at all: TypeError."""
    y, q, s = torch.zeros(3, 20), torch.zeros(20, 50, dtype=torch.uint8), torch.zeros(20, 1)
    fc4 = dict(x=torch.zeros(3, 100), q=q, scales=s, y=y, group=128)
    answer = dict(logits=torch.zeros(3, 50), given=torch.zeros(3, dtype=torch.int32), logp=torch.zeros(3))
    many = dict(x=torch.zeros(1, 100).expand(1 << 31, -1), y=torch.zeros(1, 20).expand(1 << 31, -1))
    for call, args, status in ((ctx.fc4, dict(fc4, group=1 << 31), cw.CW_ERR_UNSUPPORTED), (ctx.fc4, dict(fc4, group=1 << 70), cw.CW_ERR_UNSUPPORTED), (ctx.fc4, dict(fc4, **many), cw.CW_ERR_UNSUPPORTED),
                               (ctx.answer, dict(logits=torch.zeros(1, 50).expand(1 << 31, -1)), cw.CW_ERR_UNSUPPORTED),
                               (ctx.answer, dict(answer, scale=1e39), cw.CW_ERR_INVALID), (ctx.answer, dict(answer, scale=float("inf")), cw.CW_ERR_INVALID), (ctx.answer, dict(answer, scale=-1e300), cw.CW_ERR_INVALID)):
        with pytest.raises(cw.CwError) as e:
            call(**args)
        assert e.value.status == status and "planning-only" not in str(e.value)
    for call, args in ((ctx.fc4, dict(fc4, group=128.0)), (ctx.fc4, dict(fc4, group="128")), (ctx.answer, dict(answer, scale="1")), (ctx.answer, dict(answer, scale=None))):
        with pytest.raises(TypeError):
            call(**args)
    for top_id in (torch.zeros(3, dtype=torch.int32), torch.zeros(3, 2, 2, dtype=torch.int32)):
        with pytest.raises(ValueError):
            ctx.answer(**dict(answer, top_id=top_id, top_logp=torch.zeros(3, 2)))


def test_fc4_in_an_operator_list(ctx):
    conv, pool, soft = (T.CONV, 3, 64, 3, 3, 2, 1, 1, -1, -1, 0, 0), (T.GAVGPOOL, 64, 64, 0, 0, 1, 0, 0, -1, 0, 0, 0), (T.SOFTMAX, 10, 10, 0, 0, 1, 0, 0, -1, 2, 0, 0)
    fc4 = lambda group=32, src=1: (cw.CW_OP_FC4, 64, 10, 1, 1, 1, 0, 0, -1, src, 0, group)
    mid = ctx.model_define([conv, pool, fc4(), soft], 3, 16, 16, batch_sizes=(1, 4))
    assert ctx.model_get_ops(mid)[2] == fc4()
    weights = 64 * 3 * 9 * 2 + 10 * 32 + 10 * 2 * 2 + 10 * 2
    assert ctx.model_weight_bytes(mid) == (weights + 3) // 4 * 4 + 4 * 74
    plan = ctx.plan(mid, 4)
    assert [l["name"] for l in plan[-2:]] == ["fc4", "softmax"] and plan[-2]["flops"] == 2 * 4 * 64 * 10
    assert plan[-2]["bytes"] == 4 * 64 * 4 + 10 * (32 + 2 * 3) + 40 + 4 * 40 and plan[-2]["grid_x"] >= 1 and plan[-2]["block"] >= 64
    # fewer pages than the layer in 16 bits where it is what fills them
    wide = lambda op, g: [conv, pool, (op, 64, 100000, 1, 1, 1, 0, 0, -1, 1, 0, g), (T.SOFTMAX, 100000, 100000, 0, 0, 1, 0, 0, -1, 2, 0, 0)]
    big = cw.Context(device=-1, weight_page_bytes=16 << 20)
    try:
        assert big.model_define(wide(cw.CW_OP_FC4, 64), 3, 16, 16, batch_sizes=(1,)) == 0
    finally:
        big.destroy()
    for ops, status in (([conv, pool, fc4(0), soft], cw.CW_ERR_UNSUPPORTED), ([conv, pool, fc4(48), soft], cw.CW_ERR_UNSUPPORTED), ([conv, pool, fc4(-32), soft], cw.CW_ERR_UNSUPPORTED),
                        ([conv, pool, fc4()], cw.CW_ERR_UNSUPPORTED), ([conv, fc4(src=0), pool, soft], cw.CW_ERR_UNSUPPORTED)):
        with pytest.raises(cw.CwError) as e:
            ctx.model_define(ops, 3, 16, 16, batch_sizes=(1,))
        assert e.value.status == status


@pytest.mark.parametrize("group", [128, 1 << 20, 1 << 30, (1 << 31) - 64, (1 << 31) - 32])
@pytest.mark.parametrize("cout", [10, 1 << 20])
def test_a_group_longer_than_the_rows_is_one_group(ctx, group, cout):
    """Up to the largest one: the plan and the places of the weights are those of the shortest that holds a whole row."""
    assert refusal(ctx, cw.lib().cw_fc4, fc4_args(group=group)) == PLANNING
    ops = lambda g: [(T.CONV, 3, 64, 3, 3, 2, 1, 1, -1, -1, 0, 0), (T.GAVGPOOL, 64, 64, 0, 0, 1, 0, 0, -1, 0, 0, 0), (cw.CW_OP_FC4, 64, cout, 1, 1, 1, 0, 0, -1, 1, 0, g),
                     (T.SOFTMAX, cout, cout, 0, 0, 1, 0, 0, -1, 2, 0, 0)]
    big = cw.Context(device=-1, weight_page_bytes=64 << 20)
    try:
        short, long = (big.model_define(ops(g), 3, 16, 16, batch_sizes=(1, 4)) for g in (64, group))
        assert big.model_weight_bytes(long) == big.model_weight_bytes(short) and big.model_weight_pages(long) == big.model_weight_pages(short)
        for batch in (1, 4):
            assert big.plan(long, batch) == big.plan(short, batch)
    finally:
        big.destroy()


@pytest.mark.parametrize("classes, page, fc_pages", [(2000, 1 << 20, 2), (4000, 2 << 20, 2), (4000, 1 << 20, None)])
def test_fc4_takes_fewer_bytes_and_pages_than_the_layer_in_16_bits(classes, page, fc_pages):
    """256 features in groups of 64: 128 + 4 (2 + 1) bytes a class for 512.  The last size in 16 bits is larger than a page."""
    convs = [(T.CONV, 3, 256, 3, 3, 2, 1, 1, -1, -1, 0, 0), (T.CONV, 256, 256, 1, 1, 1, 0, 1, -1, 0, 0, 0), (T.GAVGPOOL, 256, 256, 0, 0, 1, 0, 0, -1, 1, 0, 0)]
    ops = lambda op, g: convs + [(op, 256, classes, 1, 1, 1, 0, 0, -1, 2, 0, g), (T.SOFTMAX, classes, classes, 0, 0, 1, 0, 0, -1, 3, 0, 0)]
    c = cw.Context(device=-1, weight_page_bytes=page)
    try:
        small = c.model_define(ops(cw.CW_OP_FC4, 64), 3, 16, 16, batch_sizes=(1,))
        assert c.model_weight_pages(small) == 1
        if fc_pages is None:
            with pytest.raises(cw.CwError) as e:
                c.model_define(ops(T.FC, 0), 3, 16, 16, batch_sizes=(1,))
            assert e.value.status == cw.CW_ERR_UNSUPPORTED
        else:
            large = c.model_define(ops(T.FC, 0), 3, 16, 16, batch_sizes=(1,))
            assert c.model_weight_pages(large) == fc_pages
            assert c.model_weight_bytes(large) - c.model_weight_bytes(small) == (512 - 140) * classes
    finally:
        c.destroy()
