"""What the calls over a paged cache and cw_attend refuse, on a planning-only context: every check stands before the first use of the GPU."""
import ctypes

import pytest
import torch

import paper_2006_02464_amd as cw

INVALID, UNSUPPORTED = cw.CW_ERR_INVALID, cw.CW_ERR_UNSUPPORTED
PLANNING = (INVALID, "planning-only context has no device")


@pytest.fixture()
def ctx():
    c = cw.Context(device=-1)
    yield c
    c.destroy()


def filled(kind, defaults, change):
    a = dict(defaults)
    a.update(change)
    return kind(*[a[n] for n, _ in kind._fields_])


def cache_struct(**change):
    return filled(cw.cw_cache, dict(k=4096, v=4096, k_exp=None, v_exp=None, page_stride=2 * 16 * 64, head_stride=16 * 64, token_stride=64, exp_page_stride=32, exp_head_stride=16, exp_token_stride=1,
                                    pages=10, kv_heads=2, page=16, head_dim=64, dtype=0), change)


CODES = dict(dtype=3, k_exp=4097, v_exp=4099)
ROWS = dict(k=4096, v=4096, first=4096, lengths=4096, table=4096, k_stride=128, k_head_stride=64, v_stride=128, v_head_stride=64, table_stride=5, tokens=7, sequences=3, table_pages=5, dtype=0)
ONE = dict(q=4096, y=4096, lse=4096, lengths=4096, table=4096, workspace=4096, workspace_bytes=1 << 20, q_stride=256, q_head_stride=64, y_stride=256, y_head_stride=64, table_stride=5, sequences=3, heads=4,
           table_pages=5, window=0, dtype=0, scale=0.125)
PROMPT = dict(q=4096, k=4096, v=4096, y=4096, lse=4096, first=4096, first_k=4096, q_stride=256, q_head_stride=64, k_stride=128, k_head_stride=64, v_stride=128, v_head_stride=64, y_stride=256, y_head_stride=64,
              tokens=7, keys=9, sequences=3, heads=4, kv_heads=2, head_dim=64, causal=1, window=0, dtype=0, scale=0.125)


def refusal(ctx, call, kind, defaults, change, cache=None):
    """Of the call with `change`; cache: changes of the cache, or None for a call without one."""
    if cache is not None:
        pages = cache_struct(**cache)
        defaults = dict(defaults, cache=ctypes.addressof(pages))
    st = getattr(cw.lib(), call)(ctx._h, ctypes.byref(filled(kind, defaults, change)), None)
    return st, cw.lib().cw_last_error(ctx._h).decode()


OVER_A_CACHE = [("cw_cache_write", cw.cw_cache_args, ROWS), ("cw_cache_read", cw.cw_cache_args, ROWS), ("cw_attend_one", cw.cw_attend_one_args, ONE)]


@pytest.mark.parametrize("call, kind, defaults", OVER_A_CACHE)
@pytest.mark.parametrize("change, status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=4104), INVALID), (dict(v=4098), INVALID), (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(dtype=4), INVALID),
    (dict(pages=-1), INVALID), (dict(kv_heads=0), INVALID), (dict(page=0), INVALID), (dict(page=-16), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=-64), INVALID),
    (dict(page=24), UNSUPPORTED), (dict(page=8192), UNSUPPORTED), (dict(head_dim=24), UNSUPPORTED), (dict(head_dim=272), UNSUPPORTED), (dict(kv_heads=4097), UNSUPPORTED),
    (dict(page_stride=-8), INVALID), (dict(head_stride=-8), INVALID), (dict(token_stride=-8), INVALID), (dict(page_stride=2052), INVALID), (dict(head_stride=1028), INVALID),
    (dict(token_stride=68), INVALID), (dict(page_stride=(1 << 40) + 8), INVALID), (dict(CODES, token_stride=72), INVALID), (dict(CODES, exp_page_stride=-1), INVALID),
    (dict(CODES, exp_head_stride=-1), INVALID), (dict(CODES, exp_token_stride=-1), INVALID), (dict(CODES, exp_page_stride=1 << 50), INVALID), (dict(CODES, k_exp=None), INVALID),
    (dict(CODES, v_exp=None), INVALID), (dict(k_exp=4096, v_exp=4096), INVALID), (dict(k_exp=4096), INVALID)])
def test_caches_that_are_refused(ctx, call, kind, defaults, change, status):
    st, why = refusal(ctx, call, kind, defaults, {}, change)
    assert st == status and (st, why) != PLANNING


@pytest.mark.parametrize("call, kind, defaults", OVER_A_CACHE)
@pytest.mark.parametrize("change", [{}, CODES, dict(pages=0, k=None, v=None), dict(page=1, token_stride=3), dict(page=4096, head_stride=4096 * 64, page_stride=2 * 4096 * 64),
                                    dict(head_stride=64, token_stride=128), dict(pages=1, page_stride=0), dict(head_dim=16), dict(page_stride=1 << 40)])
def test_caches_that_are_let_through(ctx, call, kind, defaults, change):
    dim = change.get("head_dim", 64)
    kv_heads = change.get("kv_heads", 2)
    assert refusal(ctx, call, kind, defaults, {}, change) == PLANNING


@pytest.mark.parametrize("change", [dict(token_stride=0), dict(token_stride=56), dict(head_stride=512), dict(page_stride=1024), dict(head_stride=0), dict(page_stride=0), dict(CODES, exp_page_stride=31),
                                    dict(CODES, exp_head_stride=8), dict(CODES, exp_token_stride=0)])
def test_written_pages_must_not_overlap(ctx, change):
    st, why = refusal(ctx, "cw_cache_write", cw.cw_cache_args, ROWS, {}, change)
    assert st == INVALID and (st, why) != PLANNING
    assert refusal(ctx, "cw_cache_read", cw.cw_cache_args, ROWS, {}, change) == PLANNING
    assert refusal(ctx, "cw_attend_one", cw.cw_attend_one_args, ONE, {}, change) == PLANNING


@pytest.mark.parametrize("call", ["cw_cache_write", "cw_cache_read"])
@pytest.mark.parametrize("change, status", [
    (dict(cache=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=4100), INVALID), (dict(v=4104), INVALID), (dict(first=4098), INVALID), (dict(lengths=None), INVALID),
    (dict(lengths=4097), INVALID), (dict(table=None), INVALID), (dict(table=4098), INVALID), (dict(k_stride=-8), INVALID), (dict(k_head_stride=-8), INVALID), (dict(v_stride=12), INVALID),
    (dict(v_head_stride=68), INVALID), (dict(table_stride=-1), INVALID), (dict(tokens=-1), INVALID), (dict(sequences=-1), INVALID), (dict(table_pages=-1), INVALID),
    (dict(tokens=(1 << 24) + 1), UNSUPPORTED), (dict(sequences=(1 << 20) + 1), UNSUPPORTED), (dict(table_pages=1 << 27), UNSUPPORTED), (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID),
    (dict(first=None), INVALID)])
def test_rows_that_are_refused(ctx, call, change, status):
    st, why = refusal(ctx, call, cw.cw_cache_args, ROWS, change, {})
    assert st == status and (st, why) != PLANNING


def test_rows_that_are_let_through(ctx):
    for change in ({}, dict(tokens=0, k=None, v=None), dict(sequences=0, lengths=None, table=None), dict(table_pages=0, table=None), dict(first=None, tokens=3), dict(dtype=2), dict(dtype=1),
                   dict(tokens=1, k_stride=3), dict(table_stride=0)):
        assert refusal(ctx, "cw_cache_write", cw.cw_cache_args, ROWS, change, {}) == PLANNING
        assert refusal(ctx, "cw_cache_read", cw.cw_cache_args, ROWS, change, {}) == PLANNING
    overlap = dict(k_stride=0)
    assert refusal(ctx, "cw_cache_write", cw.cw_cache_args, ROWS, overlap, {}) == PLANNING       # one row for all is read
    for overlap in (dict(k_stride=0), dict(v_stride=120), dict(k_head_stride=0), dict(v_head_stride=56)):
        st, why = refusal(ctx, "cw_cache_read", cw.cw_cache_args, ROWS, overlap, {})
        assert st == INVALID and (st, why) != PLANNING
    assert refusal(ctx, "cw_cache_read", cw.cw_cache_args, ROWS, dict(k_stride=64, k_head_stride=448), {}) == PLANNING    # heads ahead of tokens


@pytest.mark.parametrize("change, status", [
    (dict(cache=None), INVALID), (dict(q=None), INVALID), (dict(y=None), INVALID), (dict(q=4104), INVALID), (dict(y=4098), INVALID), (dict(lse=4098), INVALID), (dict(lengths=None), INVALID),
    (dict(lengths=4098), INVALID), (dict(table=None), INVALID), (dict(table=4099), INVALID), (dict(workspace=4104), INVALID), (dict(q_stride=-8), INVALID), (dict(q_head_stride=12), INVALID),
    (dict(y_stride=248), INVALID), (dict(y_head_stride=56), INVALID), (dict(y_head_stride=0), INVALID), (dict(y_stride=0), INVALID), (dict(table_stride=-1), INVALID), (dict(sequences=-1), INVALID),
    (dict(sequences=(1 << 20) + 1), UNSUPPORTED), (dict(heads=0), INVALID), (dict(heads=3), INVALID), (dict(heads=-2), INVALID), (dict(heads=4098), UNSUPPORTED), (dict(table_pages=-1), INVALID),
    (dict(table_pages=1 << 27), UNSUPPORTED), (dict(window=-1), INVALID), (dict(dtype=1), INVALID), (dict(dtype=2), INVALID), (dict(dtype=3), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID)])
def test_attend_one_refuses(ctx, change, status):
    st, why = refusal(ctx, "cw_attend_one", cw.cw_attend_one_args, ONE, change, {})
    assert st == status and (st, why) != PLANNING


def test_attend_one_lets_through(ctx):
    for change in ({}, dict(lse=None), dict(workspace=None, workspace_bytes=0), dict(workspace_bytes=3), dict(sequences=0, q=None, y=None, lengths=None, table=None), dict(table_pages=0, table=None),
                   dict(q_stride=0, q_head_stride=0), dict(y_stride=64, y_head_stride=192), dict(scale=-2.0), dict(scale=0.0), dict(window=2 ** 31 - 1), dict(sequences=1, y_stride=0)):
        assert refusal(ctx, "cw_attend_one", cw.cw_attend_one_args, ONE, change, {}) == PLANNING, change
    for dtype in (0, 1):
        assert refusal(ctx, "cw_attend_one", cw.cw_attend_one_args, ONE, dict(dtype=dtype), CODES) == PLANNING
    assert refusal(ctx, "cw_attend_one", cw.cw_attend_one_args, ONE, dict(dtype=1), dict(dtype=1)) == PLANNING


@pytest.mark.parametrize("change, status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(y=None), INVALID), (dict(first=None), INVALID), (dict(q=4104), INVALID), (dict(k=4104), INVALID), (dict(v=4104), INVALID),
    (dict(y=4104), INVALID), (dict(lse=4097), INVALID), (dict(first=4097), INVALID), (dict(first_k=4098), INVALID), (dict(q_stride=-8), INVALID), (dict(k_stride=4), INVALID), (dict(v_head_stride=-64), INVALID),
    (dict(k_head_stride=12), INVALID), (dict(q_head_stride=-8), INVALID), (dict(y_stride=0), INVALID), (dict(y_head_stride=32), INVALID), (dict(y_stride=128), INVALID), (dict(tokens=-1), INVALID),
    (dict(keys=-1), INVALID), (dict(sequences=-1), INVALID), (dict(tokens=(1 << 24) + 1), UNSUPPORTED), (dict(keys=(1 << 24) + 1), UNSUPPORTED), (dict(sequences=(1 << 20) + 1), UNSUPPORTED),
    (dict(heads=0), INVALID), (dict(heads=5), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=-2), INVALID), (dict(heads=4098), UNSUPPORTED), (dict(head_dim=0), INVALID), (dict(head_dim=72), UNSUPPORTED),
    (dict(head_dim=272), UNSUPPORTED), (dict(causal=2), INVALID), (dict(causal=-1), INVALID), (dict(window=-1), INVALID), (dict(causal=0, window=5), INVALID), (dict(dtype=2), INVALID), (dict(dtype=3), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(k_stride=(1 << 40) + 8), INVALID),
    (dict(k_stride=(1 << 23) + 8), UNSUPPORTED), (dict(v_stride=1 << 30), UNSUPPORTED), (dict(tokens=1 << 24, heads=128, y_stride=1 << 20, kv_heads=1), UNSUPPORTED)])
def test_attend_refuses(ctx, change, status):
    st, why = refusal(ctx, "cw_attend", cw.cw_attend_args, PROMPT, change)
    assert st == status and (st, why) != PLANNING


@pytest.mark.parametrize("change", [{}, dict(lse=None, first_k=None), dict(tokens=0, q=None, y=None), dict(keys=0, k=None, v=None), dict(sequences=0, first=None), dict(causal=0), dict(window=7),
                                    dict(q_stride=0, k_stride=0, v_stride=0, k_head_stride=0), dict(y_stride=64, y_head_stride=448), dict(heads=4096, kv_heads=4096, y_stride=1 << 18), dict(scale=-1.0),
                                    dict(dtype=1), dict(tokens=1, q_stride=1), dict(k_stride=1 << 23, v_stride=1 << 23),
                                    dict(q_stride=1 << 40), dict(keys=1, k_stride=1 << 40)])
def test_attend_lets_through(ctx, change):
    assert refusal(ctx, "cw_attend", cw.cw_attend_args, PROMPT, change) == PLANNING


def test_null_arguments(ctx):
    for name in ("cw_cache_write", "cw_cache_read", "cw_attend_one", "cw_attend"):
        call = getattr(cw.lib(), name)
        assert call(ctx._h, None, None) == INVALID and call(None, None, None) == INVALID
    assert cw.CW_ATTEND_COUNTERS <= cw.Context.attend_one_workspace_bytes() <= 32 << 20


def raises(error, call, *args, **kw):
    with pytest.raises(error) as e:
        call(*args, **kw)
    return e.value


def planning(call, *args, **kw):
    assert "planning-only" in str(raises(cw.CwError, call, *args, **kw))


def test_binding_refuses_caches_that_do_not_fit(ctx):
    """A planning-only context takes CPU tensors: they are on "its" device, -1."""
    k = torch.zeros(10, 2, 16, 64, dtype=torch.float16)
    codes, exps = torch.zeros(10, 2, 16, 64, dtype=torch.float8_e4m3fn), torch.zeros(10, 2, 16, dtype=torch.uint8)
    for args in ((k[0], k[0]), (k, k[:9]), (k, k.bfloat16()), (k, torch.zeros(10, 2, 64, 16, dtype=torch.float16).transpose(2, 3)), (k.transpose(2, 3), k.transpose(2, 3)), (codes, codes, exps),
                 (codes, codes, exps[:, :, :8], exps[:, :, :8]), (codes, codes, exps, torch.zeros(10, 16, 2, dtype=torch.uint8).transpose(1, 2))):
        raises(ValueError, ctx.cache, *args)
    for args in ((k.float(), k.float()), (k.to(torch.uint8), k.to(torch.uint8)), (codes, codes, exps.int(), exps.int())):
        raises(TypeError, ctx.cache, *args)
    held = ctx.cache(codes, codes, exps, exps)
    assert held.tensors == (codes, codes, exps, exps) and (held.kv_heads, held.head_dim) == (2, 64)


def test_binding_refuses_tensors_that_do_not_fit(ctx):
    half = torch.float16
    cache = ctx.cache(torch.zeros(10, 2, 16, 64, dtype=half), torch.zeros(10, 2, 16, 64, dtype=half))
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)
    x, table, lengths, first = torch.zeros(7, 2, 64, dtype=half), i(3, 5), i(3), i(4)
    for call, order in ((ctx.cache_write, lambda d: (d["k"], d["v"], cache)), (ctx.cache_read, None)):
        go = lambda d: (call(d["k"], d["v"], cache, d["table"], d["lengths"], first=d["first"]) if order else call(cache, d["table"], d["lengths"], d["k"], d["v"], first=d["first"]))
        ok = dict(k=x, v=x.clone(), table=table, lengths=lengths, first=first)
        planning(go, ok)
        for change in (dict(k=x[0]), dict(v=x[:6]), dict(k=torch.zeros(7, 3, 64, dtype=half)), dict(v=torch.zeros(7, 64, 2, dtype=half).transpose(1, 2)), dict(table=table[0]), dict(table=table.long()),
                       dict(table=torch.zeros(3, 5)), dict(table=i(5, 3).t()), dict(lengths=lengths[:2]), dict(lengths=lengths.long()), dict(first=first[:3]), dict(first=first.long()), dict(first=i(8)[::2])):
            raises(ValueError, go, dict(ok, **change))
        for change in (dict(k=x.float()), dict(k=x.double(), v=x.double())):
            raises(TypeError, go, dict(ok, **change))
        assert raises(cw.CwError, go, dict(ok, first=None)).status == INVALID
    q = torch.zeros(3, 4, 64, dtype=half)
    one = lambda **c: ctx.attend_one(**dict(dict(q=q, cache=cache, table=table, lengths=lengths, y=q.clone(), scale=0.1, lse=torch.zeros(3, 4), workspace=torch.zeros(64, dtype=torch.uint8)), **c))
    planning(one)
    for change in (dict(q=q[0]), dict(q=q[:2]), dict(y=q[:, :2]), dict(q=torch.zeros(3, 4, 32, dtype=half)), dict(y=torch.zeros(3, 64, 4, dtype=half).transpose(1, 2)), dict(lse=torch.zeros(3, 3)),
                   dict(lse=torch.zeros(3, 4, dtype=half)), dict(workspace=torch.zeros(64)), dict(lengths=lengths[:2]), dict(table=table.long())):
        raises(ValueError, one, **change)
    for change in (dict(q=q.float(), y=q.float()), dict(q=q.bfloat16()), dict(window=1.5), dict(scale="a"), dict(q=q.double(), y=q.double())):
        raises((TypeError, cw.CwError), one, **change)
    assert raises(cw.CwError, one, window=1 << 40).status == UNSUPPORTED
    assert raises(cw.CwError, one, scale=1e300).status == INVALID
    assert raises(cw.CwError, one, window=-1).status == INVALID
    k, q = torch.zeros(9, 2, 64, dtype=half), torch.zeros(7, 4, 64, dtype=half)
    prompt = lambda **c: ctx.attend(**dict(dict(q=q, k=k, v=k.clone(), y=q.clone(), first=first, scale=0.1, first_k=first.clone(), lse=torch.zeros(7, 4)), **c))
    planning(prompt)
    planning(prompt, causal=False)
    for change in (dict(q=q[0]), dict(k=k[0]), dict(v=k[:8]), dict(y=q[:6]), dict(k=torch.zeros(9, 2, 32, dtype=half)), dict(v=torch.zeros(9, 64, 2, dtype=half).transpose(1, 2)), dict(first=first.long()),
                   dict(first_k=first[:3]), dict(lse=torch.zeros(4, 6))):
        raises(ValueError, prompt, **change)
    for change in (dict(q=q.float()), dict(y=q.bfloat16()), dict(window=1.5)):
        raises(TypeError, prompt, **change)
    assert raises(cw.CwError, prompt, window=1 << 40).status == UNSUPPORTED
    assert raises(cw.CwError, prompt, causal=False, window=3).status == INVALID
    assert raises(cw.CwError, prompt, scale=float("nan")).status == INVALID


@pytest.mark.parametrize("call", ["cw_cache_write", "cw_cache_read"])
@pytest.mark.parametrize("tokens, let_through", [(13944699, False), (13944274, False), (13944273, True)])
def test_rows_that_32_bits_count(ctx, call, tokens, let_through):
    """Twice 77 rows a token: 2^31 - 2 of them, and one token on either side of what is left for the last workgroup's waves."""
    cache = dict(kv_heads=77, page_stride=77 * 16 * 64)
    change = dict(tokens=tokens, k_stride=77 * 64, v_stride=77 * 64)
    st, why = refusal(ctx, call, cw.cw_cache_args, ROWS, change, cache)
    assert (st, why) == PLANNING if let_through else st == UNSUPPORTED


def test_scales_at_their_end(ctx):
    """Scores are in units of ln 2: scale / ln 2 is a number of fp32."""
    for scale, status in ((2.0 ** 127, None), (-2.0 ** 127, None), (1e-45, None), (-0.0, None), (2.0 ** 127 * 1.001, INVALID), (-3.4e38, INVALID)):
        for call, kind, defaults, cache in (("cw_attend", cw.cw_attend_args, PROMPT, None), ("cw_attend_one", cw.cw_attend_one_args, ONE, {})):
            st, why = refusal(ctx, call, kind, defaults, dict(scale=scale), cache)
            assert (st, why) == PLANNING if status is None else st == status and (st, why) != PLANNING, (call, scale)


class OnGpu1(torch.Tensor):
    """A tensor that says it is on GPU 1."""

    def get_device(self):
        return 1


def test_binding_refuses_caches_of_another_gpu(ctx):
    """Pages are named by their addresses: those of another GPU than the context's must not reach it."""
    half = torch.float16
    pages = torch.zeros(10, 2, 16, 64, dtype=half).as_subclass(OnGpu1)
    raises(ValueError, ctx.cache, pages, pages)
    cache = cw.Cache(1, pages, pages, None, None)            # of a context of GPU 1
    assert cache.device == 1 and ctx.cache(torch.zeros(1, 2, 16, 64, dtype=half), torch.zeros(1, 2, 16, 64, dtype=half)).device == -1
    i = lambda *n: torch.zeros(*n, dtype=torch.int32)
    x, q = torch.zeros(3, 2, 64, dtype=half), torch.zeros(3, 4, 64, dtype=half)
    for call in (lambda: ctx.cache_write(x, x.clone(), cache, i(3, 5), i(3)), lambda: ctx.cache_read(cache, i(3, 5), i(3), x, x.clone()),
                 lambda: ctx.attend_one(q, cache, i(3, 5), i(3), q.clone(), 0.1)):
        assert "the cache is not on the context's GPU" in str(raises(ValueError, call))


def test_binding_takes_pages_that_are_laid_out_alike(ctx):
    """Strides of dimensions of one element, which torch leaves open, say nothing of the layout."""
    half, code, byte = torch.float16, torch.float8_e4m3fn, torch.uint8
    view = lambda shape, strides, dtype: torch.zeros(1 << 16, dtype=byte).view(dtype).as_strided(shape, strides)
    q, i = torch.zeros(3, 4, 64, dtype=half), lambda *n: torch.zeros(*n, dtype=torch.int32)

    def taken(*pages):
        cache = ctx.cache(*pages)
        planning(ctx.attend_one, q, cache, i(3, 5), i(3), q.clone(), 0.1)
        x = torch.zeros(3, cache.kv_heads, 64, dtype=half)
        planning(ctx.cache_write, x, x.clone(), cache, i(3, 5), i(3))
    taken(view((1, 2, 16, 64), (2048, 1024, 64, 1), half), view((1, 2, 16, 64), (1, 1024, 64, 1), half))          # one page
    taken(view((2, 1, 16, 64), (1024, 1024, 64, 1), half), view((2, 1, 16, 64), (1024, 7, 64, 1), half))          # one key head
    taken(view((2, 2, 1, 64), (128, 64, 64, 1), half), view((2, 2, 1, 64), (128, 64, 3, 1), half))                # one token a page
    taken(*(view((1, 2, 16, 64), s, code) for s in ((2048, 1024, 64, 1), (5, 1024, 64, 1))), *(view((1, 2, 16), s, byte) for s in ((32, 16, 1), (3, 16, 1))))
    taken(*(view((2, 1, 16, 64), (1024, 1024, 64, 1), code) for _ in range(2)), *(view((2, 1, 16), s, byte) for s in ((16, 16, 1), (16, 9, 1))))
    for shape, a, b in (((2, 1, 16, 64), (1024, 0, 64, 1), (2048, 0, 64, 1)), ((1, 2, 16, 64), (0, 1024, 64, 1), (0, 2048, 64, 1)), ((1, 1, 16, 64), (0, 0, 64, 1), (0, 0, 128, 1))):
        raises(ValueError, ctx.cache, view(shape, a, half), view(shape, b, half))
    raises(ValueError, ctx.cache, *(view((2, 1, 16, 64), (1024, 0, 64, 1), code) for _ in range(2)), *(view((2, 1, 16), s, byte) for s in ((16, 0, 1), (32, 0, 1))))


def test_launches_of_more_than_32_bits_of_threads(ctx):
    """A launch's threads are counted in 32 bits: calls of more are "too large" before the GPU is asked."""
    def both(call, kind, defaults, fits, beyond, cache=None):
        assert refusal(ctx, call, kind, dict(defaults, **fits), {}, cache) == PLANNING, (call, fits)
        st, why = refusal(ctx, call, kind, dict(defaults, **beyond), {}, cache)
        assert (st, why) == (UNSUPPORTED, "too large"), (call, beyond, why)
    # rows of 256 numbers, two a wave's pass, four passes: 32 a workgroup of 256
    wide = dict(kv_heads=16, head_dim=256, token_stride=256, head_stride=16 * 256, page_stride=16 * 16 * 256)
    rows = dict(ROWS, k_stride=4096, k_head_stride=256, v_stride=4096, v_head_stride=256)
    for call in ("cw_cache_write", "cw_cache_read"):
        both(call, cw.cw_cache_args, rows, dict(tokens=(1 << 24) - 1), dict(tokens=1 << 24), wide)
    # a workgroup of 256 for every sequence and key head
    prompt = dict(PROMPT, heads=16, kv_heads=16, q_stride=1024, y_stride=1024, k_stride=1024, v_stride=1024)
    both("cw_attend", cw.cw_attend_args, prompt, dict(sequences=(1 << 20) - 1), dict(sequences=1 << 20))
    both("cw_attend", cw.cw_attend_args, dict(prompt, sequences=1), dict(tokens=(1 << 24) - 200, heads=128, kv_heads=1, y_stride=8192), dict(tokens=1 << 24, heads=128, kv_heads=1, y_stride=8192))
    one = dict(ONE, heads=16, q_stride=1024, y_stride=1024)
    many = dict(kv_heads=16, page_stride=16 * 16 * 64)
    both("cw_attend_one", cw.cw_attend_one_args, dict(one, table_pages=100), dict(sequences=(1 << 20) - 1), dict(sequences=1 << 20), many)
    # of few tokens one of 64
    more = dict(kv_heads=64, page_stride=64 * 16 * 64)
    for few in (dict(table_pages=8), dict(table_pages=20), dict(table_pages=100, window=200)):
        both("cw_attend_one", cw.cw_attend_one_args, dict(one, heads=64, y_stride=4096, **few), dict(sequences=(1 << 20) - 1), dict(sequences=1 << 20), more)
        assert refusal(ctx, "cw_attend_one", cw.cw_attend_one_args, dict(one, sequences=1 << 20, **few), {}, many) == PLANNING


def test_pools_of_no_pages(ctx):
    """They have no addresses: those of 8 bits none of exponents either."""
    none = dict(pages=0, k=None, v=None)
    for call, kind, defaults in OVER_A_CACHE:
        for cache in (none, dict(CODES, **none), dict(CODES, **none, k_exp=None, v_exp=None)):
            assert refusal(ctx, call, kind, defaults, {}, cache) == PLANNING, (call, cache)
        st, why = refusal(ctx, call, kind, defaults, {}, dict(none, k_exp=4096, v_exp=4096))
        assert st == INVALID and (st, why) != PLANNING
    i, half = lambda *n: torch.zeros(*n, dtype=torch.int32), torch.float16
    codes, exps = torch.zeros(0, 2, 16, 64, dtype=torch.float8_e4m3fn), torch.zeros(0, 2, 16, dtype=torch.uint8)
    x, q = torch.zeros(3, 2, 64, dtype=half), torch.zeros(3, 4, 64, dtype=half)
    for cache in (ctx.cache(codes, codes, exps, exps), ctx.cache(codes.to(half), codes.to(half))):
        planning(ctx.cache_write, x, x.clone(), cache, i(3, 5), i(3))
        planning(ctx.attend_one, q, cache, i(3, 5), i(3), q.clone(), 0.1)
