"""CPU checks of the packed-attention boundary: exports, descriptor layout, validation, chunk plan, workspace."""
import ctypes as C
import os
import re
import subprocess

import pytest

from oracle import attention as orc
from paper_2301_08984_amd import binding as ss
from paper_2301_08984_amd import packed_binding as pb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_exports_match_header():
    text = open(os.path.join(ROOT, "include", "ss_packed.h")).read()
    assert set(re.findall(r"\b(ss_packed_\w+)\s*\(", text)) == set(pb.EXPORTS)
    for name in pb.EXPORTS:
        assert hasattr(pb.lib(), name), name


def test_struct_layout_matches_c(tmp_path):
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    fields = [f for f, _ in pb.ss_packed_desc._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ss_packed.h"\nint main(void){\n'
                   'printf("%zu\\n", sizeof(ss_packed_desc));\n'
                   + "".join(f'printf("%zu\\n", offsetof(ss_packed_desc, {f}));\n' for f in fields) + "return 0;}\n")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    out = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert out == [C.sizeof(pb.ss_packed_desc)] + [getattr(pb.ss_packed_desc, f).offset for f in fields]


@pytest.mark.parametrize("change,code", [
    (dict(Tq=0), ss.SS_ERR_BAD_SHAPE), (dict(Tk=0), ss.SS_ERR_BAD_SHAPE), (dict(n_seq=0), ss.SS_ERR_BAD_SHAPE),
    (dict(H=9), ss.SS_ERR_BAD_SHAPE), (dict(HK=0), ss.SS_ERR_BAD_SHAPE), (dict(D=60), ss.SS_ERR_BAD_SHAPE),
    (dict(D=136), ss.SS_ERR_BAD_SHAPE),   # longer than the strides
    (dict(q_stride_t=60), ss.SS_ERR_BAD_SHAPE), (dict(k_stride_h=132), ss.SS_ERR_BAD_SHAPE), (dict(y_stride_t=0), ss.SS_ERR_BAD_SHAPE),
    (dict(k_stride_t=1 << 24), ss.SS_ERR_UNSUPPORTED), (dict(q_stride_h=1 << 40), ss.SS_ERR_UNSUPPORTED),
    (dict(scale=float("nan")), ss.SS_ERR_BAD_SHAPE), (dict(scale=float("inf")), ss.SS_ERR_BAD_SHAPE),
    (dict(dtype=ss.SS_F32), ss.SS_ERR_UNSUPPORTED), (dict(flags=1), ss.SS_ERR_UNSUPPORTED), (dict(n_seq=65536), ss.SS_ERR_UNSUPPORTED),
    (dict(D=256, q_stride_h=256, k_stride_h=256, y_stride_h=256), ss.SS_ERR_UNSUPPORTED),
    (dict(lo=-1), ss.SS_ERR_BAD_RANGE), (dict(lo=2, hi=2), ss.SS_ERR_BAD_RANGE), (dict(hi=5), ss.SS_ERR_BAD_RANGE),
    (dict(k=0), ss.SS_ERR_BAD_K), (dict(k=5), ss.SS_ERR_BAD_K),
])
def test_validation(change, code):
    d = pb.make_desc(100, 3, 8, 4, 128, 0, 4, 2)
    assert pb.ss_packed_workspace_bytes(d)[0] == 0 and pb.ss_packed_workspace_bytes(d)[1] > 0
    for f, v in change.items():
        setattr(d, f, v)
    with pytest.raises(ss.SSAttnError) as e:
        pb.ss_packed_workspace_bytes(d)
    assert e.value.code == code


def test_null_pointers_and_workspace_are_refused_before_anything_is_enqueued():
    d = pb.make_desc(100, 3, 8, 4, 128, 0, 4, 2)
    a = 256  # aligned, never dereferenced: validation fails first
    need = pb.ss_packed_workspace_bytes(d)[1]

    def refused(code, call, *args):
        with pytest.raises(ss.SSAttnError) as e:
            call(d, *args)
        assert e.value.code == code, args

    for i in (0, 1, 2, 3, 5):
        args = [a, a, a, a, None, a, None, None, 0, None]
        args[i] = None
        refused(ss.SS_ERR_NULL, pb.ss_packed_fwd, *args)
    for i in (0, 1, 2, 5):
        args = [a, a, a, a, None, a, None, None, 0, None]
        args[i] = a + 8
        refused(ss.SS_ERR_BAD_SHAPE, pb.ss_packed_fwd, *args)
    good = [a, a, a, a, None, a, a, a, a, a, a, a, need, None]
    for i in (0, 1, 2, 3, 5, 6, 7, 8, 9, 10):  # 5 and 7: the output without the statistics, and the reverse
        args = list(good)
        args[i] = None
        refused(ss.SS_ERR_NULL, pb.ss_packed_bwd, *args)
    for change in (dict([(11, None)]), {11: a + 64}, {12: need - 1}):
        args = list(good)
        for i, v in change.items():
            args[i] = v
        refused(ss.SS_ERR_WORKSPACE, pb.ss_packed_bwd, *args)
    d.Tk = 90  # one array of offsets for two numbers of rows
    refused(ss.SS_ERR_BAD_SHAPE, pb.ss_packed_fwd, a, a, a, a, None, a, None, None, 0, None)
    refused(ss.SS_ERR_BAD_SHAPE, pb.ss_packed_bwd, *good)
    assert pb.lib().ss_packed_workspace_bytes(None, None, None) == ss.SS_ERR_NULL


def test_chunks_and_workspace():
    for lo, hi in ((0, 7), (2, 7), (3, 4)):
        for k in range(1, hi - lo + 1):
            d = pb.make_desc(100, 3, 14, 7, 64, lo, hi, k)
            assert [pb.ss_packed_chunk_range(d, c) for c in range(k)] == orc.chunk_ranges(lo, hi, k)
    with pytest.raises(ss.SSAttnError):
        pb.ss_packed_chunk_range(pb.make_desc(100, 3, 14, 7, 64, 0, 7, 2), 2)
    # the scratch of the backward is one chunk's
    sizes = [pb.ss_packed_workspace_bytes(pb.make_desc(8192, 20, 32, 8, 128, 0, 8, k))[1] for k in (1, 2, 4, 8)]
    assert all(a >= 1.9 * b for a, b in zip(sizes, sizes[1:])), sizes


def test_heads_and_tokens_of_a_step_that_lie_too_far_apart():
    # 28 heads and 33 tokens, each 2^24 - 8 elements apart: 1.02e9 elements, further than a lane's offset reaches
    far = (1 << 24) - 8
    d = pb.make_desc(100, 3, 28, 1, 128, 0, 1, 1)
    d.q_stride_t, d.q_stride_h = far, far
    with pytest.raises(ss.SSAttnError) as e:
        pb.ss_packed_workspace_bytes(d)
    assert e.value.code == ss.SS_ERR_UNSUPPORTED
    d.H = 26
    assert pb.ss_packed_workspace_bytes(d)[1] > 0
