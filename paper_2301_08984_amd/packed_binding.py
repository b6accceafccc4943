"""ctypes binding of the entry points declared in include/ss_packed.h, attention over packed sequences with
grouped heads (same shared library as the attention entry points).  Argument marshalling only: nothing is computed here."""
from __future__ import annotations

import ctypes as C
import math

from . import binding as _b

EXPORTS = ("ss_packed_workspace_bytes", "ss_packed_chunk_range", "ss_packed_fwd", "ss_packed_bwd")


class ss_packed_desc(C.Structure):
    _fields_ = [
        ("Tq", C.c_int32), ("Tk", C.c_int32), ("n_seq", C.c_int32), ("H", C.c_int32), ("HK", C.c_int32), ("D", C.c_int32),
        ("dtype", C.c_int32), ("scale", C.c_float),
        ("q_stride_t", C.c_int64), ("q_stride_h", C.c_int64), ("k_stride_t", C.c_int64), ("k_stride_h", C.c_int64),
        ("y_stride_t", C.c_int64), ("y_stride_h", C.c_int64),
        ("lo", C.c_int32), ("hi", C.c_int32), ("k", C.c_int32), ("flags", C.c_uint32),
    ]


_ready = False


def lib():
    global _ready
    L = _b.lib()
    if not _ready:
        P, V = C.POINTER(ss_packed_desc), C.c_void_p
        L.ss_packed_workspace_bytes.argtypes = [P, C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]
        L.ss_packed_workspace_bytes.restype = C.c_int
        L.ss_packed_chunk_range.argtypes = [P, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.ss_packed_chunk_range.restype = C.c_int
        L.ss_packed_fwd.argtypes = [P, V, V, V, V, V, V, V, V, C.c_size_t, V]
        L.ss_packed_fwd.restype = C.c_int
        L.ss_packed_bwd.argtypes = [P, V, V, V, V, V, V, V, V, V, V, V, V, C.c_size_t, V]
        L.ss_packed_bwd.restype = C.c_int
        _ready = True
    return L


def make_desc(Tq, n_seq, H, HK, D, lo, hi, k, *, Tk=None, scale=None, q_stride_t=None, q_stride_h=None, k_stride_t=None,
              k_stride_h=None, y_stride_t=None, y_stride_h=None, dtype=_b.SS_BF16, flags=0) -> ss_packed_desc:
    """Tensors packed as [T, heads, D] where no strides are given; `scale` is 1/sqrt(D) then."""
    return ss_packed_desc(Tq, Tq if Tk is None else Tk, n_seq, H, HK, D, dtype, 1.0 / math.sqrt(D) if scale is None else scale,
                          H * D if q_stride_t is None else q_stride_t, D if q_stride_h is None else q_stride_h,
                          HK * D if k_stride_t is None else k_stride_t, D if k_stride_h is None else k_stride_h,
                          H * D if y_stride_t is None else y_stride_t, D if y_stride_h is None else y_stride_h,
                          lo, hi, k, flags)


def _check(rc, where):
    if rc != _b.SS_OK:
        raise _b.SSAttnError(rc, where)


def ss_packed_workspace_bytes(desc):
    """-> (fwd_bytes, bwd_bytes); raises SSAttnError on an invalid descriptor."""
    f, b = C.c_size_t(0), C.c_size_t(0)
    _check(lib().ss_packed_workspace_bytes(C.byref(desc), C.byref(f), C.byref(b)), "ss_packed_workspace_bytes")
    return f.value, b.value


def ss_packed_chunk_range(desc, c):
    lo, hi = C.c_int32(0), C.c_int32(0)
    _check(lib().ss_packed_chunk_range(C.byref(desc), c, C.byref(lo), C.byref(hi)), "ss_packed_chunk_range")
    return lo.value, hi.value


def ss_packed_fwd(desc, Q, K, V, cu_q, cu_k, Y, lse, workspace, workspace_bytes, stream):
    p = _b._ptr
    _check(lib().ss_packed_fwd(C.byref(desc), p(Q), p(K), p(V), p(cu_q), p(cu_k), p(Y), p(lse), p(workspace), workspace_bytes,
                               stream), "ss_packed_fwd")


def ss_packed_bwd(desc, Q, K, V, cu_q, cu_k, Y, dY, lse, dQ, dK, dV, workspace, workspace_bytes, stream):
    p = _b._ptr
    _check(lib().ss_packed_bwd(C.byref(desc), p(Q), p(K), p(V), p(cu_q), p(cu_k), p(Y), p(dY), p(lse), p(dQ), p(dK), p(dV),
                               p(workspace), workspace_bytes, stream), "ss_packed_bwd")
