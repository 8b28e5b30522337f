"""ctypes binding of include/clockwork_exec.h: same names, argument marshalling
only.  Every step of the path runs in the library's HIP kernels."""
import ctypes
import os
import struct
from ctypes import (POINTER, Structure, byref, c_char, c_char_p, c_float, c_int32,
                    c_int64, c_size_t, c_uint32, c_uint64, c_void_p)

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libclockwork_exec.so")

CW_OK = 0
CW_ERR_INVALID, CW_ERR_HIP, CW_ERR_NO_MEMORY, CW_ERR_NOT_LOADED = -1, -2, -3, -4
CW_ERR_ALREADY_LOADED, CW_ERR_NO_INPUT, CW_ERR_BAD_BATCH, CW_ERR_BUSY = -5, -6, -7, -8
CW_ERR_UNSUPPORTED, CW_ERR_NO_SLOT, CW_ERR_TOO_LATE, CW_ERR_TIMEOUT = -9, -10, -11, -12
CW_OP_CONV, CW_OP_MAXPOOL, CW_OP_GAVGPOOL, CW_OP_FC, CW_OP_SOFTMAX, CW_OP_CONCAT = 0, 1, 2, 3, 4, 5
CW_OP_FC4 = 6
CW_DTYPE_FP16, CW_DTYPE_BF16, CW_DTYPE_FP32, CW_DTYPE_E4M3 = 0, 1, 2, 3
CW_ANSWER_MOST_TOP, CW_ANSWER_COUNTERS = 64, 1024
CW_CACHE_MOST_PAGE, CW_ATTEND_MOST_DIM, CW_ATTEND_COUNTERS = 4096, 256, 65536
DTYPES = {"fp16": CW_DTYPE_FP16, "bf16": CW_DTYPE_BF16}
CONV_TILES = {"128x128": 0, "128x64": 1, "64x64": 2, "64x32": 3, "32x64": 4, "32x32": 5,
              "128x64w2": 6, "64x128w2": 7, "256x64": 8, "128x128w8": 9,
              "128x64k128": 10, "64x64k128": 11, "64x32k128": 12, "32x64k128": 13, "32x32k128": 14,
              "128x64k128g2": 15, "64x64k128g2": 16, "64x64k128g4": 17, "64x32k128g4": 18, "32x64k128g4": 19,
              "32x32k128g4": 20, "32x32k128g8": 21, "128x64g2": 22, "64x64g2": 23, "32x32g4": 24,
              "256x128w8": 25, "128x256w8": 26, "256x256w8": 27, "256x128": 28}


class cw_op(Structure):
    _fields_ = [(n, c_int32) for n in ("op", "cin", "cout", "kh", "kw", "stride", "pad",
                                        "relu", "residual_from", "input_from", "pad_w", "groups")]


class cw_config(Structure):
    _fields_ = [("device", c_int32), ("workspace_bytes", c_size_t), ("io_bytes", c_size_t),
                ("weight_pool_bytes", c_size_t), ("load_staging_bytes", c_size_t), ("weight_page_bytes", c_size_t)]


class cw_fc4_args(Structure):
    _fields_ = [(n, c_void_p) for n in ("x", "q", "scales", "zeros", "bias", "y")] + \
               [(n, c_int64) for n in ("x_stride", "q_stride", "scale_stride", "zero_stride", "y_stride")] + \
               [(n, c_int32) for n in ("rows", "cin", "cout", "group", "x_dtype", "scale_dtype", "y_dtype")]


class cw_answer_args(Structure):
    _fields_ = [(n, c_void_p) for n in ("logits", "given", "logp", "rank", "entropy", "top_id", "top_logp", "workspace")] + \
               [("workspace_bytes", c_size_t), ("stride", c_int64)] + \
               [(n, c_int32) for n in ("rows", "classes", "top", "dtype")] + [("scale", c_float)]


class cw_cache(Structure):
    _fields_ = [(n, c_void_p) for n in ("k", "v", "k_exp", "v_exp")] + \
               [(n, c_int64) for n in ("page_stride", "head_stride", "token_stride", "exp_page_stride", "exp_head_stride", "exp_token_stride")] + \
               [(n, c_int32) for n in ("pages", "kv_heads", "page", "head_dim", "dtype")]


class cw_cache_args(Structure):
    _fields_ = [(n, c_void_p) for n in ("cache", "k", "v", "first", "lengths", "table")] + \
               [(n, c_int64) for n in ("k_stride", "k_head_stride", "v_stride", "v_head_stride", "table_stride")] + \
               [(n, c_int32) for n in ("tokens", "sequences", "table_pages", "dtype")]


class cw_attend_one_args(Structure):
    _fields_ = [(n, c_void_p) for n in ("cache", "q", "y", "lse", "lengths", "table", "workspace")] + \
               [("workspace_bytes", c_size_t)] + \
               [(n, c_int64) for n in ("q_stride", "q_head_stride", "y_stride", "y_head_stride", "table_stride")] + \
               [(n, c_int32) for n in ("sequences", "heads", "table_pages", "window", "dtype")] + [("scale", c_float)]


class cw_attend_args(Structure):
    _fields_ = [(n, c_void_p) for n in ("q", "k", "v", "y", "lse", "first", "first_k")] + \
               [(n, c_int64) for n in ("q_stride", "q_head_stride", "k_stride", "k_head_stride", "v_stride", "v_head_stride", "y_stride", "y_head_stride")] + \
               [(n, c_int32) for n in ("tokens", "keys", "sequences", "heads", "kv_heads", "head_dim", "causal", "window", "dtype")] + [("scale", c_float)]


class cw_profile(Structure):
    _fields_ = [("n", c_uint32), ("p50_us", c_float), ("p99_us", c_float), ("p999_us", c_float),
                ("min_us", c_float), ("max_us", c_float), ("mean_us", c_float), ("p9999_us", c_float)]


class cw_launch_info(Structure):
    _fields_ = [("op_index", c_int32), ("fused_op", c_int32), ("proj_op", c_int32), ("pair_op", c_int32), ("kind", c_int32), ("grid_x", c_int32), ("grid_y", c_int32),
                ("grid_z", c_int32), ("block", c_int32), ("tile_m", c_int32), ("tile_n", c_int32),
                ("tile_k", c_int32), ("split_k", c_int32), ("conv_tile", c_int32), ("wave_groups", c_int32), ("next_op", c_int32), ("panels", c_int32), ("gemm_m", c_int64), ("gemm_n", c_int64), ("gemm_k", c_int64),
                ("bytes", c_int64), ("flops", c_int64), ("name", c_char * 48)]


class cw_action(Structure):
    _fields_ = [("id", c_int64), ("type", c_int32), ("model_id", c_int32), ("batch", c_int32), ("earliest_ns", c_uint64),
                ("latest_ns", c_uint64), ("host_in", c_void_p), ("host_in_bytes", c_size_t), ("host_probs", c_void_p),
                ("host_logits", c_void_p)]


class cw_result(Structure):
    _fields_ = [("id", c_int64), ("type", c_int32), ("status", c_int32), ("begin_ns", c_uint64), ("end_ns", c_uint64),
                ("device_ns", c_uint64)]


CW_ACTION_LOAD, CW_ACTION_UNLOAD, CW_ACTION_INFER = 1, 2, 3

# name -> (restype, argtypes); every symbol the header declares
SIGNATURES = {
    "cw_create": (c_int32, [POINTER(c_void_p), POINTER(cw_config)]),
    "cw_destroy": (c_int32, [c_void_p]),
    "cw_model_define": (c_int32, [c_void_p, POINTER(cw_op), c_int32, c_int32, c_int32, c_int32,
                                  POINTER(c_int32), c_int32, c_int32, POINTER(c_int32)]),
    "cw_model_define_resnet": (c_int32, [c_void_p, c_int32, c_int32, c_int32, c_int32, POINTER(c_int32)]),
    "cw_model_get_ops": (c_int32, [c_void_p, c_int32, POINTER(cw_op), c_int32, POINTER(c_int32)]),
    "cw_model_weight_bytes": (c_size_t, [c_void_p, c_int32]),
    "cw_model_workspace_bytes": (c_size_t, [c_void_p, c_int32, c_int32]),
    "cw_load_weights": (c_int32, [c_void_p, c_int32, c_void_p, c_size_t, c_void_p]),
    "cw_load_weights_begin": (c_int32, [c_void_p, c_int32, c_void_p, c_size_t, c_void_p, POINTER(c_void_p)]),
    "cw_load_weights_record": (c_int32, [c_void_p, c_void_p]),
    "cw_load_weights_end": (c_int32, [c_void_p, c_void_p]),
    "cw_load_weights_release": (None, [c_void_p]),
    "cw_unload_weights": (c_int32, [c_void_p, c_int32]),
    "cw_weight_pool_free": (c_size_t, [c_void_p]),
    "cw_weight_pages_free": (c_int32, [c_void_p]),
    "cw_context_device": (c_int32, [c_void_p]),
    "cw_worker_create": (c_int32, [c_void_p, POINTER(c_int32), POINTER(c_void_p)]),
    "cw_worker_destroy": (c_int32, [c_void_p]),
    "cw_worker_now_ns": (c_uint64, []),
    "cw_worker_submit": (c_int32, [c_void_p, POINTER(cw_action)]),
    "cw_worker_next_result": (c_int32, [c_void_p, POINTER(cw_result), c_uint64]),
    "cw_worker_profile": (c_int32, [c_void_p, c_int32, c_int32, c_int32, POINTER(c_uint32), POINTER(c_uint64), POINTER(c_uint64)]),
    "cw_model_weight_pages": (c_int32, [c_void_p, c_int32]),
    "cw_input": (c_int32, [c_void_p, c_int32, c_int32, c_void_p, POINTER(c_int32), c_void_p]),
    "cw_exec": (c_int32, [c_void_p, c_int32, c_int32, c_int32, c_void_p]),
    "cw_exec_static": (c_int32, [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p]),
    "cw_exec_static_capacity": (c_size_t, []),
    "cw_output": (c_int32, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p]),
    "cw_output_answer": (c_int32, [c_void_p, c_int32, c_void_p, c_int32, c_float, c_void_p, c_void_p]),
    "cw_answer_bytes": (c_size_t, [c_int32, c_int32]),
    "cw_slot_batch": (c_int32, [c_void_p, c_int32]),
    "cw_fc4": (c_int32, [c_void_p, c_void_p, c_void_p]),
    "cw_answer": (c_int32, [c_void_p, c_void_p, c_void_p]),
    "cw_answer_workspace_bytes": (c_size_t, []),
    "cw_cache_write": (c_int32, [c_void_p, c_void_p, c_void_p]),
    "cw_cache_read": (c_int32, [c_void_p, c_void_p, c_void_p]),
    "cw_attend_one": (c_int32, [c_void_p, c_void_p, c_void_p]),
    "cw_attend_one_workspace_bytes": (c_size_t, []),
    "cw_attend": (c_int32, [c_void_p, c_void_p, c_void_p]),
    "cw_release": (c_int32, [c_void_p, c_int32]),
    "cw_exec_duration_ns": (c_int32, [c_void_p, c_int32, POINTER(c_uint64)]),
    "cw_profile_measure": (c_int32, [c_void_p, c_int32, c_int32, c_int32, c_uint32, POINTER(cw_profile), c_void_p]),
    "cw_profile_get": (c_int32, [c_void_p, c_int32, c_int32, POINTER(cw_profile)]),
    "cw_plan_num_launches": (c_int32, [c_void_p, c_int32, c_int32]),
    "cw_plan_launch_info": (c_int32, [c_void_p, c_int32, c_int32, c_int32, POINTER(cw_launch_info)]),
    "cw_plan_launch_ahead": (c_int32, [c_void_p, c_int32, c_int32, c_int32, POINTER(c_int32), POINTER(c_int64)]),
    "cw_plan_launch_joined": (c_int32, [c_void_p, c_int32, c_int32, c_int32]),
    "cw_plan_launch_tail": (c_int32, [c_void_p, c_int32, c_int32, c_int32]),
    "cw_plan_launch_loaders": (c_int32, [c_void_p, c_int32, c_int32, c_int32]),
    "cw_plan_launch_issued": (c_int32, [c_void_p, c_int32, c_int32, c_int32, POINTER(cw_launch_info)]),
    "cw_exec_timed_launches": (c_int32, [c_void_p, c_int32, c_int32, c_int32, c_int32, c_void_p, c_void_p]),
    "cw_debug_read_op": (c_int32, [c_void_p, c_int32, c_int32, c_int32, c_void_p, c_size_t]),
    "cw_set_debug_keep": (c_int32, [c_void_p, c_int32]),
    "cw_set_debug_keep_joined": (c_int32, [c_void_p, c_int32]),
    "cw_set_plan_override": (c_int32, [c_void_p, c_int32, c_int32]),
    "cw_set_plan_table": (c_int32, [c_void_p, c_void_p, c_int32]),
    "cw_set_fusion": (c_int32, [c_void_p, c_int32]),
    "cw_set_pair_launches": (c_int32, [c_void_p, c_int32]),
    "cw_set_panels": (c_int32, [c_void_p, c_int32]),
    "cw_set_fusion_third": (c_int32, [c_void_p, c_int32]),
    "cw_set_fusion_pool": (c_int32, [c_void_p, c_int32]),
    "cw_set_fusion_dw": (c_int32, [c_void_p, c_int32]),
    "cw_set_fc_softmax": (c_int32, [c_void_p, c_int32]),
    "cw_set_winograd": (c_int32, [c_void_p, c_int32]),
    "cw_set_resident": (c_int32, [c_void_p, c_int32]),
    "cw_set_use_graphs": (c_int32, [c_void_p, c_int32]),
    "cw_set_wait_launches": (c_int32, [c_void_p, c_int32]),
    "cw_output_by_launch": (c_int32, [c_void_p, c_void_p, c_size_t]),
    "cw_strerror": (c_char_p, [c_int32]),
    "cw_last_error": (c_char_p, [c_void_p]),
}

_lib = None
_int32 = _float32 = None    # torch's


def lib():
    """The loaded library.  Builds it only if no built library exists; fails
    loudly if it cannot be had (there is no other implementation to fall to)."""
    global _lib
    if _lib is None:
        # PyTorch ships its own HIP runtime under the same soname.  Importing it first makes the
        # dynamic loader hand that one copy to this library too; loaded the other way round the
        # process would hold two HIP runtimes, and the second one fails to initialise.
        import torch  # noqa: F401
        if not os.path.exists(LIB_PATH):
            from . import build as _build
            _build.build()
        l = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype, fn.argtypes = res, args
        global _int32, _float32
        _int32, _float32 = torch.int32, torch.float32
        _lib = l
    return _lib


class CwError(RuntimeError):
    def __init__(self, status, detail=""):
        self.status = status
        name = lib().cw_strerror(status).decode()
        super().__init__("%s (%d)%s" % (name, status, (": " + detail) if detail else ""))


def _ptr(x):
    """Host address of a numpy array / torch CPU tensor / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return c_void_p(x)
    if isinstance(x, np.ndarray):
        assert x.flags["C_CONTIGUOUS"]
        return c_void_p(x.ctypes.data)
    if hasattr(x, "data_ptr"):
        assert x.is_contiguous()
        return c_void_p(x.data_ptr())
    raise TypeError(type(x))


def _packed(args):
    """What packs the fields of a Structure `args` into bytes: 0.2 us, where the Structure takes 0.8 of calls that last a few."""
    fields = struct.Struct("@" + "".join({c_void_p: "P", c_size_t: "N", c_int64: "q", c_int32: "i", c_float: "f"}[t] for _, t in args._fields_) + "0q")
    assert fields.size == ctypes.sizeof(args)
    return fields.pack


_pack_fc4, _pack_answer = _packed(cw_fc4_args), _packed(cw_answer_args)
_pack_cache_args, _pack_attend_one, _pack_attend = _packed(cw_cache_args), _packed(cw_attend_one_args), _packed(cw_attend_args)


def _refused(error, **numbers):
    """The error for numbers that do not fit their fields, in the library's terms."""
    for name, number in numbers.items():
        if not hasattr(number, "__index__") and not (name == "scale" and hasattr(number, "__float__")):
            return TypeError("%s: %r" % (name, number))
    if isinstance(error, OverflowError):
        return CwError(CW_ERR_INVALID, "scale must be finite and positive")
    return CwError(CW_ERR_UNSUPPORTED, "too large: " + ", ".join("%s %s" % n for n in numbers.items()))


class _Types(dict):
    """CW_DTYPE_* of a torch dtype."""

    def __missing__(self, dtype):
        if not self:
            import torch
            self.update({torch.float16: CW_DTYPE_FP16, torch.bfloat16: CW_DTYPE_BF16, torch.float32: CW_DTYPE_FP32})
            return self[dtype]
        raise TypeError("%s is no element type of this call" % dtype)


class _PageTypes(dict):
    """CW_DTYPE_* of a torch dtype that a cache's pages have."""

    def __missing__(self, dtype):
        if not self:
            import torch
            self.update({torch.float16: CW_DTYPE_FP16, torch.bfloat16: CW_DTYPE_BF16, torch.float8_e4m3fn: CW_DTYPE_E4M3})
            return self[dtype]
        raise TypeError("%s is no type of a cache's pages" % dtype)


_element_codes, _page_codes = _Types(), _PageTypes()
_vector_types = {}   # names of torch dtypes


def _matrix(t, what, device, rows, cols):
    """(address, row stride) of a matrix on GPU `device` whose rows are contiguous."""
    if t.get_device() != device:
        raise ValueError("%s is not on the context's GPU" % what)
    if t.shape != (rows, cols):
        raise ValueError("%s is %s, not %s" % (what, tuple(t.shape), (rows, cols)))
    row, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s: elements of a row must be contiguous" % what)
    return t.data_ptr(), row


def _vector(t, what, device, count, kind):
    """Address of a contiguous tensor of `count` elements of the type `kind` there, or 0."""
    if t is None:
        return 0
    if t.get_device() != device:
        raise ValueError("%s is not on the context's GPU" % what)
    dtype = t.dtype
    if dtype not in _vector_types:
        _vector_types[dtype] = str(dtype)
    if t.numel() != count or _vector_types[dtype] != kind or not t.is_contiguous():
        raise ValueError("%s must be %d contiguous elements of %s" % (what, count, kind))
    return t.data_ptr()


def _heads(t, what, device, rows, heads, shape=None):
    """(address, row stride, head stride) of [rows][heads][head_dim], which is `shape` if that is not known yet, on GPU `device` whose last elements are contiguous."""
    if t.get_device() != device:
        raise ValueError("%s is not on the context's GPU" % what)
    if shape is not None and t.shape != shape:
        raise ValueError("%s is %s, not %s" % (what, tuple(t.shape), tuple(shape)))
    row, head, step = t.stride()
    if step != 1:
        raise ValueError("%s: numbers of a head must be contiguous" % what)
    return t.data_ptr(), row if rows > 1 else 0, head if heads > 1 else 0


def _ints(t, what, device, count):
    """Address of `count` contiguous elements of int32 there."""
    if t.dtype is _int32 and t.get_device() == device and t.numel() == count and t.is_contiguous():
        return t.data_ptr()
    return _vector(t, what, device, count, "torch.int32")


def _floats(t, what, device, count):
    """The same of fp32, or 0."""
    if t is None:
        return 0
    if t.dtype is _float32 and t.get_device() == device and t.numel() == count and t.is_contiguous():
        return t.data_ptr()
    return _vector(t, what, device, count, "torch.float32")


def _table(table, device):
    """(address of the table, its row stride, sequences, pages a row)."""
    shape = table.shape
    if len(shape) != 2:
        raise ValueError("table is %s, not (sequences, pages)" % (tuple(shape),))
    if table.dtype is not _int32:
        raise ValueError("table holds int32")
    if table.get_device() != device:
        raise ValueError("table is not on the context's GPU")
    sequences, pages = shape
    row, step = table.stride()
    if step != 1 and pages > 1:
        raise ValueError("table: elements of a row must be contiguous")
    return table.data_ptr(), row if sequences > 1 else 0, sequences, pages


def _on(stream):
    """Handle of a stream as a number."""
    return 0 if stream is None else stream if isinstance(stream, int) else stream.cuda_stream


def _strides(t):
    """Of the dimensions, 0 of those of one element: torch leaves these open."""
    return tuple(step if n > 1 else 0 for n, step in zip(t.shape, t.stride()))


class Cache:
    """Pages of keys and values as the calls over them take them: made by Context.cache, holds the tensors that it names."""

    def __init__(self, device, k, v, k_exp, v_exp):
        if k.dim() != 4:
            raise ValueError("k is %s, not (pages, kv_heads, page, head_dim)" % (tuple(k.shape),))
        strides = _strides(k)
        if v.shape != k.shape or _strides(v) != strides or v.dtype != k.dtype:
            raise ValueError("k and v are laid out differently")
        pages, kv_heads, page, head_dim = k.shape
        if strides[3] != 1 and head_dim > 1:
            raise ValueError("numbers of a head must be contiguous")
        if (k_exp is None) != (v_exp is None):
            raise ValueError("exponents of both keys and values, or of neither")
        exps = (0, 0, 0)
        if k_exp is not None:
            if k_exp.shape != k.shape[:3] or v_exp.shape != k.shape[:3] or _strides(k_exp) != _strides(v_exp):
                raise ValueError("k_exp and v_exp must be %s and laid out alike" % (tuple(k.shape[:3]),))
            if str(k_exp.dtype) != "torch.uint8" or str(v_exp.dtype) != "torch.uint8":
                raise TypeError("exponents are bytes")
            exps = _strides(k_exp)
        for t in (k, v, k_exp, v_exp):
            if t is not None and t.get_device() != device:
                raise ValueError("the cache is not on the context's GPU")
        at = [t.data_ptr() if t is not None else None for t in (k, v, k_exp, v_exp)]
        try:
            fields = at + [int(n) for n in (*strides[:3], *exps)]
            if not all(0 <= n < 1 << 31 for n in k.shape):
                raise CwError(CW_ERR_UNSUPPORTED, "too large")
            self._struct = cw_cache(*fields, pages, kv_heads, page, head_dim, _page_codes[k.dtype])
        except OverflowError:
            raise CwError(CW_ERR_UNSUPPORTED, "too large") from None
        self.tensors = (k, v, k_exp, v_exp)
        self.device, self.kv_heads, self.head_dim = device, kv_heads, head_dim
        self.address = ctypes.addressof(self._struct)


def _host(x, what):
    """(address, bytes, element type by name) of contiguous host memory: a numpy array, a CPU tensor."""
    if isinstance(x, np.ndarray):
        here, whole, nbytes, kind = True, x.flags["C_CONTIGUOUS"], x.nbytes, x.dtype.name if x.dtype.isnative else x.dtype.str
    elif hasattr(x, "data_ptr"):
        here, whole, nbytes, kind = x.device.type == "cpu", x.is_contiguous(), x.numel() * x.itemsize, str(x.dtype)[len("torch."):]
    else:
        raise TypeError("%s: %s is no array" % (what, type(x).__name__))
    if not here or not whole:
        raise ValueError("%s must be contiguous host memory" % what)
    return _ptr(x), nbytes, kind


def _stream(s):
    if s is None:
        return None
    if isinstance(s, int):
        return c_void_p(s)
    return c_void_p(s.cuda_stream)  # torch.cuda.Stream


class Context:
    """One worker-GPU.  Methods carry the C names without the ``cw_`` prefix and
    raise :class:`CwError` on a negative status."""

    def __init__(self, device=0, workspace_bytes=512 << 20, io_bytes=512 << 20,
                 weight_pool_bytes=1 << 30, load_staging_bytes=256 << 20, weight_page_bytes=0):
        self._h = c_void_p()
        cfg = cw_config(device, workspace_bytes, io_bytes, weight_pool_bytes, load_staging_bytes, weight_page_bytes)
        st = lib().cw_create(byref(self._h), byref(cfg))
        if st != CW_OK:
            self._h = c_void_p()
            raise CwError(st, "cw_create: " + lib().cw_last_error(None).decode())
        self._device = lib().cw_context_device(self._h)

    def _check(self, st):
        if st < 0:
            raise CwError(st, lib().cw_last_error(self._h).decode())
        return st

    def destroy(self):
        if self._h:
            lib().cw_destroy(self._h)
            self._h = c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # -- models
    def model_define(self, ops, in_c, in_h, in_w, batch_sizes=(1, 2, 4, 8, 16), dtype="fp16"):
        arr = (cw_op * len(ops))(*[cw_op(*[int(v) for v in o]) for o in ops])
        bs = (c_int32 * len(batch_sizes))(*batch_sizes)
        mid = c_int32(-1)
        self._check(lib().cw_model_define(self._h, arr, len(ops), in_c, in_h, in_w, bs,
                                          len(batch_sizes), DTYPES[dtype], byref(mid)))
        return mid.value

    def model_define_resnet(self, depth, in_h, in_w, dtype="fp16"):
        mid = c_int32(-1)
        self._check(lib().cw_model_define_resnet(self._h, depth, in_h, in_w, DTYPES[dtype], byref(mid)))
        return mid.value

    def model_get_ops(self, model_id):
        n = c_int32(0)
        self._check(lib().cw_model_get_ops(self._h, model_id, None, 0, byref(n)))
        arr = (cw_op * n.value)()
        self._check(lib().cw_model_get_ops(self._h, model_id, arr, n.value, byref(n)))
        return [tuple(getattr(o, f) for f, _ in cw_op._fields_) for o in arr]

    def model_weight_bytes(self, model_id):
        return lib().cw_model_weight_bytes(self._h, model_id)

    def model_workspace_bytes(self, model_id, batch):
        return lib().cw_model_workspace_bytes(self._h, model_id, batch)

    # -- LOAD / UNLOAD
    def load_weights(self, model_id, host_blob, stream=None):
        nbytes = host_blob.nbytes if isinstance(host_blob, np.ndarray) else host_blob.numel() * host_blob.element_size()
        self._check(lib().cw_load_weights(self._h, model_id, _ptr(host_blob), nbytes, _stream(stream)))

    def load_weights_begin(self, model_id, host_blob, stream=None):
        """First step of a LOAD in steps; returns the handle the other three steps take."""
        nbytes = host_blob.nbytes if isinstance(host_blob, np.ndarray) else host_blob.numel() * host_blob.element_size()
        pending = c_void_p()
        self._check(lib().cw_load_weights_begin(self._h, model_id, _ptr(host_blob), nbytes, _stream(stream), ctypes.byref(pending)))
        return pending

    def load_weights_record(self, pending):
        self._check(lib().cw_load_weights_record(self._h, pending))

    def load_weights_end(self, pending):
        self._check(lib().cw_load_weights_end(self._h, pending))

    def load_weights_release(self, pending):
        lib().cw_load_weights_release(pending)

    def unload_weights(self, model_id):
        self._check(lib().cw_unload_weights(self._h, model_id))

    def weight_pool_free(self):
        return lib().cw_weight_pool_free(self._h)

    def weight_pages_free(self):
        return self._check(lib().cw_weight_pages_free(self._h))

    def model_weight_pages(self, model_id):
        return self._check(lib().cw_model_weight_pages(self._h, model_id))

    # -- INFER
    def input(self, model_id, batch, host_nchw, stream=None):
        slot = c_int32(-1)
        self._check(lib().cw_input(self._h, model_id, batch, _ptr(host_nchw), byref(slot), _stream(stream)))
        return slot.value

    def exec(self, model_id, batch, slot, stream=None):
        self._check(lib().cw_exec(self._h, model_id, batch, slot, _stream(stream)))

    def exec_static(self, model_id, batch, dev_input, dev_logits, dev_probs, stream=None):
        """dev_*: device tensors (anything with data_ptr()) or raw device addresses."""
        self._check(lib().cw_exec_static(self._h, model_id, batch, _ptr(dev_input), _ptr(dev_logits), _ptr(dev_probs),
                                         _stream(stream)))

    @staticmethod
    def exec_static_capacity():
        return lib().cw_exec_static_capacity()

    def output(self, slot, host_probs, host_logits=None, stream=None):
        self._check(lib().cw_output(self._h, slot, _ptr(host_probs), _ptr(host_logits), _stream(stream)))

    def output_answer(self, slot, host_answer, given=None, top=0, scale=1.0, stream=None):
        """host_answer: answer_bytes(batch, top) bytes; split_answer() names their parts once `stream` has been synchronised.
        given: int32, one for each sample.  Both are host memory that stays until then: arrays, CPU tensors or, unchecked, addresses."""
        batch = lib().cw_slot_batch(self._h, slot)   # none: the call says so
        if host_answer is None or isinstance(host_answer, int):
            to = _ptr(host_answer)
        else:
            to, nbytes, _ = _host(host_answer, "host_answer")
            if isinstance(host_answer, np.ndarray) and not host_answer.flags["WRITEABLE"]:
                raise ValueError("host_answer cannot be written")
            if nbytes < self.answer_bytes(batch, top):
                raise ValueError("host_answer has %d bytes, the answer %d" % (nbytes, self.answer_bytes(batch, top)))
        if given is None or isinstance(given, int):
            classes = _ptr(given)
        else:
            classes, nbytes, kind = _host(given, "given")
            if kind != "int32" or (batch >= 0 and nbytes != 4 * batch):
                raise ValueError("given must be %s contiguous elements of int32" % (batch if batch >= 0 else "a sample's"))
        self._check(lib().cw_output_answer(self._h, slot, classes, top, scale, to, _stream(stream)))

    def slot_batch(self, slot):
        return self._check(lib().cw_slot_batch(self._h, slot))

    @staticmethod
    def answer_bytes(batch, top):
        return lib().cw_answer_bytes(batch, top)

    @staticmethod
    def split_answer(host_answer, batch, top):
        """The parts of an answer in host memory (a numpy array or a CPU tensor), as views."""
        flat = host_answer if isinstance(host_answer, np.ndarray) else host_answer.numpy()
        w = flat.reshape(-1).view(np.uint8)[:batch * (12 + 8 * top)].view(np.int32)
        return {"logp": w[:batch].view(np.float32), "rank": w[batch:2 * batch], "entropy": w[2 * batch:3 * batch].view(np.float32),
                "top_id": w[3 * batch:(3 + top) * batch].reshape(batch, top),
                "top_logp": w[(3 + top) * batch:].view(np.float32).reshape(batch, top)}

    # -- single operators over device tensors
    def fc4(self, x, q, scales, y, group, zeros=None, bias=None, stream=None):
        """y[rows][cout] = bias + x[rows][cin] times the 4-bit weights q[cout][ceil(cin / 2)] (uint8) with scales and zeros
        [cout][ceil(cin / group)]: torch tensors on the context's GPU; y is written."""
        rows, cin = x.shape
        cout = y.shape[1] if y.dim() == 2 else -1
        if group < 1:
            raise ValueError("group must be positive")
        groups, on, code = (cin + group - 1) // group, self._device, _element_codes
        xp, xs = _matrix(x, "x", on, rows, cin)
        qp, qs = _matrix(q, "q", on, cout, (cin + 1) // 2)
        sp, ss = _matrix(scales, "scales", on, cout, groups)
        zp, zs = _matrix(zeros, "zeros", on, cout, groups) if zeros is not None else (0, 0)
        yp, ys = _matrix(y, "y", on, rows, cout)
        if q.itemsize != 1 or (zeros is not None and zeros.itemsize != 1):
            raise TypeError("q and zeros hold bytes")
        try:
            args = _pack_fc4(xp, qp, sp, zp, _vector(bias, "bias", on, cout, "torch.float32"), yp, xs, qs, ss, zs, ys,
                             rows, cin, cout, group, code[x.dtype], code[scales.dtype], code[y.dtype])
        except (struct.error, OverflowError) as e:
            raise _refused(e, rows=rows, cin=cin, cout=cout, group=group) from None
        self._check(lib().cw_fc4(self._h, args, _stream(stream)))

    def answer(self, logits, given=None, logp=None, rank=None, entropy=None, top_id=None, top_logp=None, scale=1.0, workspace=None,
               stream=None):
        """The answer of every row of logits[rows][classes]: torch tensors on the context's GPU, given and rank int32, the others
        fp32; those that are not None are written, top_id and top_logp [rows][top].  workspace: uint8, zeros before its first call."""
        rows, classes = logits.shape
        on = self._device
        lp, ls = _matrix(logits, "logits", on, rows, classes)
        if top_id is not None and top_id.dim() != 2:
            raise ValueError("top_id is %s, not (rows, top)" % (tuple(top_id.shape),))
        top = top_id.shape[1] if top_id is not None else 0
        space = workspace.numel() if workspace is not None else 0
        try:
            args = _pack_answer(
                lp, _vector(given, "given", on, rows, "torch.int32"), _vector(logp, "logp", on, rows, "torch.float32"),
                _vector(rank, "rank", on, rows, "torch.int32"), _vector(entropy, "entropy", on, rows, "torch.float32"),
                _vector(top_id, "top_id", on, rows * top, "torch.int32"), _vector(top_logp, "top_logp", on, rows * top, "torch.float32"),
                _vector(workspace, "workspace", on, space, "torch.uint8"), space, ls,
                rows, classes, top, _element_codes[logits.dtype], scale)
        except (struct.error, OverflowError) as e:
            raise _refused(e, rows=rows, classes=classes, top=top, scale=scale) from None
        self._check(lib().cw_answer(self._h, args, _stream(stream)))

    @staticmethod
    def answer_workspace_bytes():
        return lib().cw_answer_workspace_bytes()

    # -- a paged cache of keys and values, and attention
    def cache(self, k, v, k_exp=None, v_exp=None):
        """Names pages: k, v [pages][kv_heads][page][head_dim] in fp16, bf16 or float8_e4m3fn, the last with exponents [pages][kv_heads][page] (uint8).  Kept
        as long as the pages are, for contexts of their GPU; what the library refuses of them the calls that take it tell."""
        return Cache(self._device, k, v, k_exp, v_exp)

    def _cache_rows(self, call, cache, k, v, table, lengths, first, stream):
        shape, heads = k.shape, cache.kv_heads
        if len(shape) != 3 or shape[1] != heads or shape[2] != cache.head_dim:
            raise ValueError("k is %s, not (tokens, %d, %d)" % (tuple(shape), heads, cache.head_dim))
        dtype, on, tokens = k.dtype, self._device, shape[0]
        if cache.device != on:
            raise ValueError("the cache is not on the context's GPU")
        if dtype is not v.dtype:
            raise TypeError("k and v are of different types")
        kp, ks, kh = _heads(k, "k", on, tokens, heads)
        vp, vs, vh = _heads(v, "v", on, tokens, heads, shape)
        tp, ts, sequences, pages = _table(table, on)
        try:
            args = _pack_cache_args(cache.address, kp, vp, 0 if first is None else _ints(first, "first", on, sequences + 1), _ints(lengths, "lengths", on, sequences), tp,
                                    ks, kh, vs, vh, ts, tokens, sequences, pages, _element_codes[dtype])
        except (struct.error, OverflowError) as e:
            raise _refused(e, tokens=tokens, sequences=sequences, pages=pages) from None
        status = call(self._h, args, _on(stream))
        if status < 0:
            self._check(status)

    def cache_write(self, k, v, cache, table, lengths, first=None, stream=None):
        """Writes rows of k and v [tokens][kv_heads][head_dim] to the pages of `cache` as the last tokens of their sequences: rows first[s]..first[s + 1] - 1 of
        sequence s, that has lengths[s] tokens with them and its pages in table[s]; without `first` a row each.  torch tensors on the context's GPU, integers int32."""
        self._cache_rows(_lib.cw_cache_write, cache, k, v, table, lengths, first, stream)

    def cache_read(self, cache, table, lengths, k, v, first=None, stream=None):
        """Reads the same rows back into k and v."""
        self._cache_rows(_lib.cw_cache_read, cache, k, v, table, lengths, first, stream)

    def attend_one(self, q, cache, table, lengths, y, scale, window=0, lse=None, workspace=None, stream=None):
        """y[sequences][heads][head_dim] = attention of q, a token of each sequence, over the lengths[s] tokens (the last `window`) in the pages table[s] of
        `cache`; lse [sequences][heads] fp32 is written if there is one.  workspace: uint8, zeros before its first call.  A table is best as wide as the
        longest sequence needs: how sequences are shared goes by its width."""
        on, dtype, shape = self._device, q.dtype, q.shape
        if cache.device != on:
            raise ValueError("the cache is not on the context's GPU")
        tp, ts, sequences, pages = _table(table, on)
        if len(shape) != 3 or shape[0] != sequences or shape[2] != cache.head_dim:
            raise ValueError("q is %s, not (%d, heads, %d)" % (tuple(shape), sequences, cache.head_dim))
        if y.dtype is not dtype:
            raise TypeError("q and y are of different types")
        heads = shape[1]
        qp, qs, qh = _heads(q, "q", on, sequences, heads)
        yp, ys, yh = _heads(y, "y", on, sequences, heads, shape)
        space = workspace.numel() if workspace is not None else 0
        try:
            args = _pack_attend_one(cache.address, qp, yp, _floats(lse, "lse", on, sequences * heads), _ints(lengths, "lengths", on, sequences), tp,
                                    _vector(workspace, "workspace", on, space, "torch.uint8"), space, qs, qh, ys, yh, ts,
                                    sequences, heads, pages, window, _element_codes[dtype], scale)
        except (struct.error, OverflowError) as e:
            raise _refused(e, sequences=sequences, heads=heads, window=window, scale=scale) from None
        status = _lib.cw_attend_one(self._h, args, _on(stream))
        if status < 0:
            self._check(status)

    @staticmethod
    def attend_one_workspace_bytes():
        return lib().cw_attend_one_workspace_bytes()

    def attend(self, q, k, v, y, first, scale, first_k=None, causal=True, window=0, lse=None, stream=None):
        """y[tokens][heads][head_dim] = attention of packed queries: rows first[s]..first[s + 1] - 1 of q over rows first_k[s]..first_k[s + 1] - 1 (the same, without
        first_k) of k and v [keys][kv_heads][head_dim]; lse [tokens][heads] fp32 is written if there is one."""
        dtype, on, shape, shape_k, sequences = q.dtype, self._device, q.shape, k.shape, first.numel() - 1
        if len(shape) != 3 or len(shape_k) != 3 or shape[2] != shape_k[2]:
            raise ValueError("q is %s, k %s, not (tokens, heads, head_dim)" % (tuple(shape), tuple(shape_k)))
        if k.dtype is not dtype or v.dtype is not dtype or y.dtype is not dtype:
            raise TypeError("q, k, v and y are of different types")
        tokens, heads, head_dim = shape
        keys, kv_heads, _ = shape_k
        qp, qs, qh = _heads(q, "q", on, tokens, heads)
        kp, ks, kh = _heads(k, "k", on, keys, kv_heads)
        vp, vs, vh = _heads(v, "v", on, keys, kv_heads, shape_k)
        yp, ys, yh = _heads(y, "y", on, tokens, heads, shape)
        try:
            args = _pack_attend(qp, kp, vp, yp, _floats(lse, "lse", on, tokens * heads), _ints(first, "first", on, sequences + 1),
                                0 if first_k is None else _ints(first_k, "first_k", on, sequences + 1), qs, qh, ks, kh, vs, vh, ys, yh,
                                tokens, keys, sequences, heads, kv_heads, head_dim, causal, window, _element_codes[dtype], scale)
        except (struct.error, OverflowError) as e:
            raise _refused(e, tokens=tokens, keys=keys, sequences=sequences, window=window, scale=scale) from None
        status = _lib.cw_attend(self._h, args, _on(stream))
        if status < 0:
            self._check(status)

    def release(self, slot):
        self._check(lib().cw_release(self._h, slot))

    def exec_duration_ns(self, slot):
        ns = c_uint64(0)
        self._check(lib().cw_exec_duration_ns(self._h, slot, byref(ns)))
        return ns.value

    # -- profile
    def profile_measure(self, model_id, batch, repeats, want_samples=False, slot=-1):
        prof = cw_profile()
        samples = np.empty(repeats, np.float32) if want_samples else None
        self._check(lib().cw_profile_measure(self._h, model_id, batch, slot, repeats, byref(prof), _ptr(samples)))
        d = {f: getattr(prof, f) for f, _ in cw_profile._fields_}
        return (d, samples) if want_samples else d

    def profile_get(self, model_id, batch):
        prof = cw_profile()
        self._check(lib().cw_profile_get(self._h, model_id, batch, byref(prof)))
        return {f: getattr(prof, f) for f, _ in cw_profile._fields_}

    # -- introspection
    def plan_num_launches(self, model_id, batch):
        return self._check(lib().cw_plan_num_launches(self._h, model_id, batch))

    def plan_launch_info(self, model_id, batch, index):
        return self._launch_info(lib().cw_plan_launch_info, model_id, batch, index)

    def _launch_info(self, call, model_id, batch, index):
        info = cw_launch_info()
        self._check(call(self._h, model_id, batch, index, byref(info)))
        d = {f: getattr(info, f) for f, _ in cw_launch_info._fields_}
        d["name"] = d["name"].decode()
        return d

    def plan_launch_ahead(self, model_id, batch, index):
        """(workgroups, bytes) that launch `index` spends on reading a later launch's weights ahead."""
        wgs, nbytes = c_int32(0), c_int64(0)
        self._check(lib().cw_plan_launch_ahead(self._h, model_id, batch, index, byref(wgs), byref(nbytes)))
        return wgs.value, nbytes.value

    def plan_launch_joined(self, model_id, batch, index):
        """Whether plan entry `index` has no launch of its own: the first convolution's launch computes it (cast, max pool),
        the FC's (average pool), a depthwise convolution's (the 1x1 in front of it), a 3x3's (the 1x1 of a densely connected
        layer) or that of a bottleneck tail's last layer."""
        return bool(self._check(lib().cw_plan_launch_joined(self._h, model_id, batch, index)))

    def plan_launch_tail(self, model_id, batch, index):
        """Layers of the bottleneck tail that entry `index` launches (2 or 3), 1 for one that a later entry's launch computes, 0 for any other."""
        return self._check(lib().cw_plan_launch_tail(self._h, model_id, batch, index))

    def plan_launch_loaders(self, model_id, batch, index):
        """Threads of a workgroup of entry `index`, as a launch of its own, that only load (beside its `block`)."""
        return self._check(lib().cw_plan_launch_loaders(self._h, model_id, batch, index))

    def plan_launch_issued(self, model_id, batch, index):
        """What EXEC issues for plan entry `index`: the work of joined entries stands with the entry that launches it."""
        return self._launch_info(lib().cw_plan_launch_issued, model_id, batch, index)

    def plan(self, model_id, batch):
        return [self.plan_launch_info(model_id, batch, i) for i in range(self.plan_num_launches(model_id, batch))]

    def issued(self, model_id, batch):
        """The launches of an EXEC: (entry of the plan, what it issues)."""
        return [(i, self.plan_launch_issued(model_id, batch, i)) for i in range(self.plan_num_launches(model_id, batch))
                if not self.plan_launch_joined(model_id, batch, i)]

    def exec_timed_launches(self, model_id, batch, slot, stream=None, inner=1):
        us = np.empty(self.plan_num_launches(model_id, batch), np.float32)
        self._check(lib().cw_exec_timed_launches(self._h, model_id, batch, slot, inner, _ptr(us), _stream(stream)))
        return us

    def debug_read_op(self, model_id, batch, op_index, shape):
        out = np.empty(shape, np.float32)
        self._check(lib().cw_debug_read_op(self._h, model_id, batch, op_index, _ptr(out), out.size))
        return out

    def set_debug_keep(self, keep, joined=False):
        """joined: the launches that compute several convolutions stay as they are without retention."""
        self._check(lib().cw_set_debug_keep(self._h, int(keep)))
        self._check(lib().cw_set_debug_keep_joined(self._h, int(joined)))

    def set_use_graphs(self, on):
        self._check(lib().cw_set_use_graphs(self._h, int(on)))

    def set_wait_launches(self, us=-1):
        self._check(lib().cw_set_wait_launches(self._h, int(us)))

    def output_by_launch(self, host, nbytes):
        """Whether OUTPUT writes `nbytes` at the address `host` by a launch, not by a copy of the runtime."""
        return bool(self._check(lib().cw_output_by_launch(self._h, host, nbytes)))

    def set_plan_override(self, conv_tile=-1, split_k=0):
        if isinstance(conv_tile, str):
            conv_tile = CONV_TILES[conv_tile]
        self._check(lib().cw_set_plan_override(self._h, conv_tile, split_k))

    def set_pair_launches(self, on):
        self._check(lib().cw_set_pair_launches(self._h, int(on)))

    def set_fc_softmax(self, on):
        self._check(lib().cw_set_fc_softmax(self._h, int(on)))

    def set_fusion_third(self, on):
        self._check(lib().cw_set_fusion_third(self._h, int(on)))

    def set_fusion_pool(self, on):
        self._check(lib().cw_set_fusion_pool(self._h, int(on)))

    def set_fusion_dw(self, on):
        self._check(lib().cw_set_fusion_dw(self._h, int(on)))

    def set_panels(self, on):
        self._check(lib().cw_set_panels(self._h, int(on)))

    def set_resident(self, on):
        self._check(lib().cw_set_resident(self._h, int(on)))

    def set_winograd(self, on):
        self._check(lib().cw_set_winograd(self._h, int(on)))

    def set_fusion(self, on):
        self._check(lib().cw_set_fusion(self._h, int(on)))

    def set_plan_table(self, rows):
        """rows: iterable of (M, N, K, kh, stride, conv_tile, split_k); empty removes the table."""
        arr = np.ascontiguousarray(np.array([[CONV_TILES[v] if isinstance(v, str) else v for v in r] for r in rows],
                                            dtype=np.int32).reshape(-1, 7))
        self._check(lib().cw_set_plan_table(self._h, _ptr(arr) if len(arr) else None, len(arr)))


__all__ = [n for n in dir() if n.startswith("CW_") or n.startswith("cw_")] + [
    "Cache", "Context", "CwError", "lib", "LIB_PATH", "SIGNATURES", "DTYPES", "CONV_TILES"]


class Executors:
    """The worker's executors over one Context (C names without the ``cw_worker_`` prefix).  Host
    buffers of submitted actions are kept alive here until their results have been fetched."""

    def __init__(self, ctx, cores=None):
        self._ctx = ctx
        self._h = c_void_p()
        arr = (c_int32 * 5)(*cores) if cores is not None else None
        st = lib().cw_worker_create(ctx._h, arr, byref(self._h))
        if st < 0:
            raise CwError(st, "cw_worker_create")
        self._keep = {}

    @staticmethod
    def now_ns():
        return lib().cw_worker_now_ns()

    def submit(self, action_id, type, model_id, earliest_ns, latest_ns, batch=0, host_in=None, host_probs=None, host_logits=None):
        nbytes = 0
        if host_in is not None:
            nbytes = host_in.nbytes if isinstance(host_in, np.ndarray) else host_in.numel() * host_in.element_size()
        a = cw_action(action_id, type, model_id, batch, earliest_ns, latest_ns, _ptr(host_in), nbytes, _ptr(host_probs), _ptr(host_logits))
        self._keep[action_id] = (host_in, host_probs, host_logits)
        st = lib().cw_worker_submit(self._h, byref(a))
        if st < 0:
            self._keep.pop(action_id, None)
            raise CwError(st, "cw_worker_submit")

    def next_result(self, timeout_s=5.0):
        """dict of the next finished action, or None after the time-out."""
        r = cw_result()
        st = lib().cw_worker_next_result(self._h, byref(r), int(timeout_s * 1e9))
        if st == CW_ERR_TIMEOUT:
            return None
        if st < 0:
            raise CwError(st, "cw_worker_next_result")
        self._keep.pop(r.id, None)
        return {f: getattr(r, f) for f, _ in cw_result._fields_}

    def profile(self, type, model_id, batch=0):
        n, mean, mx = c_uint32(0), c_uint64(0), c_uint64(0)
        st = lib().cw_worker_profile(self._h, type, model_id, batch, byref(n), byref(mean), byref(mx))
        if st < 0:
            raise CwError(st, "cw_worker_profile")
        return {"n": n.value, "mean_ns": mean.value, "max_ns": mx.value}

    def destroy(self):
        if self._h:
            lib().cw_worker_destroy(self._h)
            self._h = c_void_p()
            self._keep.clear()
