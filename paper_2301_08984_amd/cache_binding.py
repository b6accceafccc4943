"""ctypes binding of the entry points declared in include/ss_cache.h, the paged cache of keys and values and the attention
over it (same shared library as the attention entry points).  Argument marshalling only: nothing is computed here."""
from __future__ import annotations

import ctypes as C
import math

from . import binding as _b

SS_CACHE_BF16, SS_CACHE_FP8, SS_CACHE_INT8 = 0, 1, 2
EXPORTS = ("ss_cache_bytes", "ss_cache_write", "ss_cache_read", "ss_cache_attn_workspace_bytes", "ss_cache_attn")


class ss_cache_desc(C.Structure):
    _fields_ = [
        ("n_pages", C.c_int32), ("page", C.c_int32), ("HK", C.c_int32), ("D", C.c_int32), ("format", C.c_int32),
        ("n_seq", C.c_int32), ("max_pages", C.c_int32),
    ]


class ss_cache_attn_desc(C.Structure):
    _fields_ = [
        ("T", C.c_int32), ("H", C.c_int32), ("max_new", C.c_int32), ("scale", C.c_float),
        ("q_stride_t", C.c_int64), ("q_stride_h", C.c_int64), ("y_stride_t", C.c_int64), ("y_stride_h", C.c_int64),
    ]


_ready = False


def lib():
    global _ready
    L = _b.lib()
    if not _ready:
        P, A, V, I64 = C.POINTER(ss_cache_desc), C.POINTER(ss_cache_attn_desc), C.c_void_p, C.c_int64
        L.ss_cache_bytes.argtypes = [P, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.ss_cache_bytes.restype = C.c_int
        L.ss_cache_write.argtypes = [P, C.c_int32, V, V, I64, I64, V, V, V, V, V, V, V, V]
        L.ss_cache_write.restype = C.c_int
        L.ss_cache_read.argtypes = [P, C.c_int32, V, V, V, V, V, V, V, V, V, I64, I64, V]
        L.ss_cache_read.restype = C.c_int
        L.ss_cache_attn_workspace_bytes.argtypes = [P, A, C.POINTER(C.c_size_t)]
        L.ss_cache_attn_workspace_bytes.restype = C.c_int
        L.ss_cache_attn.argtypes = [P, A, V, V, V, V, V, V, V, V, V, V, V, V, C.c_size_t, V]
        L.ss_cache_attn.restype = C.c_int
        _ready = True
    return L


def make_desc(n_pages, page, HK, D, format, n_seq, max_pages) -> ss_cache_desc:
    return ss_cache_desc(n_pages, page, HK, D, format, n_seq, max_pages)


def make_attn_desc(T, H, max_new, D, *, scale=None, q_stride_t=None, q_stride_h=None, y_stride_t=None,
                   y_stride_h=None) -> ss_cache_attn_desc:
    """Tensors packed as [T, H, D] where no strides are given; `scale` is 1/sqrt(D) then."""
    return ss_cache_attn_desc(T, H, max_new, 1.0 / math.sqrt(D) if scale is None else scale,
                              H * D if q_stride_t is None else q_stride_t, D if q_stride_h is None else q_stride_h,
                              H * D if y_stride_t is None else y_stride_t, D if y_stride_h is None else y_stride_h)


def _check(rc, where):
    if rc != _b.SS_OK:
        raise _b.SSAttnError(rc, where)


def ss_cache_bytes(desc):
    """-> (bytes of one code array, of one scale array); raises SSAttnError on an invalid descriptor."""
    c, s = C.c_size_t(0), C.c_size_t(0)
    _check(lib().ss_cache_bytes(C.byref(desc), C.byref(c), C.byref(s)), "ss_cache_bytes")
    return c.value, s.value


def ss_cache_write(desc, T, K, V, stride_t, stride_h, cu, start, table, k_codes, k_scales, v_codes, v_scales, stream):
    p = _b._ptr
    _check(lib().ss_cache_write(C.byref(desc), T, p(K), p(V), stride_t, stride_h, p(cu), p(start), p(table), p(k_codes),
                                p(k_scales), p(v_codes), p(v_scales), stream), "ss_cache_write")


def ss_cache_read(desc, T, cu, start, table, k_codes, k_scales, v_codes, v_scales, K, V, stride_t, stride_h, stream):
    p = _b._ptr
    _check(lib().ss_cache_read(C.byref(desc), T, p(cu), p(start), p(table), p(k_codes), p(k_scales), p(v_codes), p(v_scales),
                               p(K), p(V), stride_t, stride_h, stream), "ss_cache_read")


def ss_cache_attn_workspace_bytes(desc, attn):
    b = C.c_size_t(0)
    _check(lib().ss_cache_attn_workspace_bytes(C.byref(desc), C.byref(attn), C.byref(b)), "ss_cache_attn_workspace_bytes")
    return b.value


def ss_cache_attn(desc, attn, Q, cu, lens, tree, table, k_codes, k_scales, v_codes, v_scales, Y, lse, workspace,
                  workspace_bytes, stream):
    p = _b._ptr
    _check(lib().ss_cache_attn(C.byref(desc), C.byref(attn), p(Q), p(cu), p(lens), p(tree), p(table), p(k_codes), p(k_scales),
                               p(v_codes), p(v_scales), p(Y), p(lse), p(workspace), workspace_bytes, stream), "ss_cache_attn")
