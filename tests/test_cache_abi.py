"""CPU checks of the cache's boundary: exports, descriptor layouts, validation, sizes, and the rule that finds a row."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import cache as oc
from paper_2301_08984_amd import binding as ss
from paper_2301_08984_amd import cache_binding as cb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_exports_match_header():
    text = open(os.path.join(ROOT, "include", "ss_cache.h")).read()
    assert set(re.findall(r"\bint (ss_cache_\w+)\s*\(", text)) == set(cb.EXPORTS)
    for name in cb.EXPORTS:
        assert hasattr(cb.lib(), name), name


@pytest.mark.parametrize("struct", [cb.ss_cache_desc, cb.ss_cache_attn_desc])
def test_struct_layout_matches_c(struct, tmp_path):
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    fields, name = [f for f, _ in struct._fields_], struct.__name__
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ss_cache.h"\nint main(void){\n'
                   f'printf("%zu\\n", sizeof({name}));\n'
                   + "".join(f'printf("%zu\\n", offsetof({name}, {f}));\n' for f in fields) + "return 0;}\n")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    out = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert out == [C.sizeof(struct)] + [getattr(struct, f).offset for f in fields]


@pytest.mark.parametrize("change,code", [
    (dict(n_pages=0), ss.SS_ERR_BAD_SHAPE), (dict(HK=0), ss.SS_ERR_BAD_SHAPE), (dict(n_seq=0), ss.SS_ERR_BAD_SHAPE),
    (dict(max_pages=0), ss.SS_ERR_BAD_SHAPE), (dict(page=0), ss.SS_ERR_BAD_SHAPE),
    (dict(page=4), ss.SS_ERR_UNSUPPORTED), (dict(page=48), ss.SS_ERR_UNSUPPORTED), (dict(page=2048), ss.SS_ERR_UNSUPPORTED),
    (dict(D=96), ss.SS_ERR_UNSUPPORTED), (dict(format=3), ss.SS_ERR_UNSUPPORTED), (dict(max_pages=1 << 28), ss.SS_ERR_UNSUPPORTED),
    (dict(n_seq=65536), ss.SS_ERR_UNSUPPORTED), (dict(n_pages=1 << 30, page=1024, HK=512), ss.SS_ERR_UNSUPPORTED),
])
def test_validation(change, code):
    d = cb.make_desc(40, 16, 4, 128, cb.SS_CACHE_FP8, 3, 10)
    assert cb.ss_cache_bytes(d) == (40 * 16 * 4 * 128, 40 * 16 * 4 * 4)
    assert cb.ss_cache_bytes(cb.make_desc(40, 16, 4, 128, cb.SS_CACHE_BF16, 3, 10)) == (40 * 16 * 4 * 256, 0)
    for f, v in change.items():
        setattr(d, f, v)
    a = cb.make_attn_desc(3, 8, 1, 128)
    one = 256
    for call in (lambda: cb.ss_cache_bytes(d), lambda: cb.ss_cache_attn_workspace_bytes(d, a),
                 lambda: cb.ss_cache_write(d, 3, one, one, 1024, 128, one, None, one, one, one, one, one, None),
                 lambda: cb.ss_cache_read(d, 3, one, None, one, one, one, one, one, one, one, 1024, 128, None)):
        with pytest.raises(ss.SSAttnError) as e:
            call()
        assert e.value.code == code


@pytest.mark.parametrize("change,code", [
    (dict(T=0), ss.SS_ERR_BAD_SHAPE), (dict(H=6), ss.SS_ERR_BAD_SHAPE), (dict(H=0), ss.SS_ERR_BAD_SHAPE), (dict(max_new=0), ss.SS_ERR_BAD_SHAPE),
    (dict(max_new=65), ss.SS_ERR_UNSUPPORTED), (dict(scale=float("inf")), ss.SS_ERR_BAD_SHAPE),
    (dict(q_stride_t=64), ss.SS_ERR_BAD_SHAPE), (dict(y_stride_h=132), ss.SS_ERR_BAD_SHAPE),
])
def test_attention_validation(change, code):
    d, a = cb.make_desc(40, 16, 4, 128, cb.SS_CACHE_FP8, 3, 10), cb.make_attn_desc(3, 8, 1, 128)
    need = cb.ss_cache_attn_workspace_bytes(d, a)
    for f, v in change.items():
        setattr(a, f, v)
    one = 256
    for call in (lambda: cb.ss_cache_attn_workspace_bytes(d, a),
                 lambda: cb.ss_cache_attn(d, a, one, one, one, None, one, one, one, one, one, one, None, one, need, None)):
        with pytest.raises(ss.SSAttnError) as e:
            call()
        assert e.value.code == code


def test_null_pointers_are_refused():
    d, a, one = cb.make_desc(40, 16, 4, 128, cb.SS_CACHE_INT8, 3, 10), cb.make_attn_desc(3, 8, 1, 128), 256
    need = cb.ss_cache_attn_workspace_bytes(d, a)

    def refused(code, call, args, at, value):
        args = list(args)
        args[at] = value
        with pytest.raises(ss.SSAttnError) as e:
            call(*args)
        assert e.value.code == code, (call.__name__, at)

    write = [d, 3, one, one, 512, 128, one, None, one, one, one, one, one, None]
    read = [d, 3, one, None, one, one, one, one, one, one, one, 512, 128, None]
    attn = [d, a, one, one, one, None, one, one, one, one, one, one, None, one, need, None]
    for call, args, null, pointers in ((cb.ss_cache_write, write, (2, 3, 6, 8, 9, 10, 11, 12), (2, 3, 9, 11)),
                                       (cb.ss_cache_read, read, (2, 4, 5, 6, 7, 8, 9, 10), (5, 7, 9, 10)),
                                       (cb.ss_cache_attn, attn, (2, 3, 4, 6, 7, 8, 9, 10, 11), (2, 7, 9, 11))):
        for at in null:
            refused(ss.SS_ERR_NULL, call, args, at, None)
        for at in pointers:
            refused(ss.SS_ERR_BAD_SHAPE, call, args, at, one + 8)
    refused(ss.SS_ERR_BAD_SHAPE, cb.ss_cache_write, write, 1, 0)
    refused(ss.SS_ERR_BAD_SHAPE, cb.ss_cache_write, write, 4, 100)
    refused(ss.SS_ERR_BAD_SHAPE, cb.ss_cache_read, read, 12, 120)
    if need:
        refused(ss.SS_ERR_WORKSPACE, cb.ss_cache_attn, attn, 13, None)
        refused(ss.SS_ERR_WORKSPACE, cb.ss_cache_attn, attn, 14, need - 1)
        refused(ss.SS_ERR_WORKSPACE, cb.ss_cache_attn, attn, 13, one + 64)


def test_rows_are_found_as_the_definition_says(tmp_path):
    """The function that the kernels find a row with, on the host: bad pages, positions outside the table, page borders, row
    numbers beyond 32 bits."""
    src, obj, exe = tmp_path / "find.cpp", tmp_path / "find.o", tmp_path / "find"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "cache.h"\n'
                   'int main(int c, char** v) {\n'
                   '  const int32_t table[] = {7, -1, 40, 39, 0, 1 << 30, 5, 5, (int32_t)0x80000000, 3};  // two lines of 5\n'
                   '  long long b, pos;\n'
                   '  while (std::scanf("%lld %lld", &b, &pos) == 2) {\n'
                   '    const int at = ssa::cache_page(table, 40, 4, 5, (int)b, pos);\n'
                   '    std::printf("%d %lld\\n", at, at < 0 ? -1ll : (long long)ssa::cache_row(at, 4, 3, 2, pos));\n'
                   '  }\n'
                   '  std::printf("%lld\\n", (long long)ssa::cache_row(30000000, 10, 96, 95, 1023));\n'
                   '  return 0;\n}\n')
    csrc = os.path.join(ROOT, "paper_2301_08984_amd", "csrc")
    subprocess.check_call(["hipcc", "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-I", csrc, "-c", str(src), "-o", str(obj)])
    subprocess.check_call(["g++", str(obj), "-o", str(exe), "-no-pie", "-Wl,--unresolved-symbols=ignore-all"])
    table = np.array([[7, -1, 40, 39, 0], [1 << 30, 5, 5, -2 ** 31, 3]])
    asked = [(b, pos) for b in (0, 1) for pos in list(range(-3, 84)) + [-2 ** 31, 2 ** 31, 2 ** 40]]
    out = subprocess.run([str(exe)], input="\n".join(f"{b} {p}" for b, p in asked), capture_output=True, text=True, check=True).stdout.split("\n")
    for (b, pos), line in zip(asked, out):
        at = oc.find(table, 40, 16, b, pos)
        page, row = (int(x) for x in line.split())
        assert (page, row) == ((-1, -1) if at is None else (at[0], (at[0] * 3 + 2) * 16 + at[1])), (b, pos)
    assert int(out[len(asked)]) == (30000000 * 96 + 95) * 1024 + 1023


def _line(lens, new, G, whole=False):
    """Units of every run of a key head's line, in order: (sequence, group of rows, units)."""
    out = []
    for b, (n_keys, n) in enumerate(zip(lens, new)):
        many = n * G > 64
        units = 1 if whole else max(1, -(-n_keys // (64 if many else 128)))
        out += [(b, g, units) for g in range(-(-n * G // 128) if many else min(n, 1))]
    return out


@pytest.mark.parametrize("seed", range(8))
def test_pieces_cover_the_line_and_parts_have_slots_of_their_own(seed):
    """The arithmetic by which the kernels deal out keys and find each other's parts."""
    rng = np.random.default_rng(seed)
    for _ in range(60):
        G, n_seq, pieces = int(rng.integers(1, 20)), int(rng.integers(1, 40)), int(rng.integers(1, 65))
        lens, new = rng.integers(0, 4000, n_seq) * rng.integers(0, 2, n_seq), rng.integers(0, 40, n_seq)
        runs = _line(lens, new, G)
        total = sum(u for _, _, u in runs)
        if not total:
            continue
        each = max(2, -(-total // pieces))
        assert -(-total // each) <= pieces
        written, first = {}, 0
        starts = []
        for b, g, units in runs:
            starts.append(first)
            first += units
        for piece in range(pieces):  # as the attention's kernels go
            u, stop = piece * each, min(piece * each + each, total)
            while u < stop:
                i = max(k for k, s in enumerate(starts) if s <= u)
                at, units = u - starts[i], runs[i][2]
                take = min(units - at, stop - u)
                if take < units:
                    slot = 2 * piece + (starts[i] > piece * each)
                    assert slot < 2 * pieces and slot not in written
                    written[slot] = (i, at, take)
                u += take
        for i, (b, g, units) in enumerate(runs):  # as the joining kernel does
            begin = starts[i]
            piece, parts = begin // each, (begin + units - 1) // each - begin // each + 1
            if parts == 1:
                assert all(w[0] != i for w in written.values())
                continue
            slots = [2 * piece + (begin > piece * each)] + [2 * (piece + x) + (begin > (piece + x) * each) for x in range(1, parts)]
            assert slots[1:] == [2 * (piece + x) for x in range(1, parts)]
            got = [written.pop(s) for s in slots]
            assert [w[0] for w in got] == [i] * parts and sum(w[2] for w in got) == units
            assert [w[1] for w in got] == list(np.cumsum([0] + [w[2] for w in got[:-1]]))
        assert not written
