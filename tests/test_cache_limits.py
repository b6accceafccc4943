"""The keys that a piece's units cover, by the function that the kernels use, up to the longest sequences that a table has room for."""
import os
import subprocess

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_pieces_of_a_run_cover_its_keys(tmp_path):
    src, obj, exe = tmp_path / "span.cpp", tmp_path / "span.o", tmp_path / "span"
    src.write_text('#include <cstdio>\n#include "cache.h"\n'
                   'int main() {\n'
                   '  int at, take, units, sh, len;\n'
                   '  while (std::scanf("%d %d %d %d %d", &at, &take, &units, &sh, &len) == 5) {\n'
                   '    const ssa::CacheSpan s = ssa::cache_span(at, take, units, sh, len);\n'
                   '    std::printf("%d %d\\n", s.begin, s.end);\n'
                   '  }\n  return 0;\n}\n')
    csrc = os.path.join(ROOT, "paper_2301_08984_amd", "csrc")
    subprocess.check_call(["hipcc", "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xarch_host", "-fsanitize=undefined",
                           "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", csrc, "-c", str(src), "-o", str(obj)])
    subprocess.check_call(["hipcc", str(obj), "-fsanitize=undefined", "-o", str(exe)])
    rng = np.random.default_rng(0)
    asked, want = [(0, 1, 1, 7, 0)], [(0, 0)]  # no key: one unit all the same
    for length in [1, 63, 64, 65, 127, 128, 129, 4000, 2 ** 31 - 1, 2 ** 31 - 8, 2 ** 31 - 64, 2 ** 31 - 127, 2 ** 31 - 128, 2 ** 31 - 129] + list(rng.integers(1, 2 ** 31, 40)):
        length = int(length)
        for sh in (6, 7):
            units = (length - 1 >> sh) + 1
            cuts = sorted({0, units, *(int(x) for x in rng.integers(0, units + 1, 4)), max(units - 1, 0), max(units - 2, 0)})
            for a, b in zip(cuts[:-1], cuts[1:]):
                asked.append((a, b - a, units, sh, length))
                want.append((a << sh, min(b << sh, length)))
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, x)) for x in asked), capture_output=True, text=True)
    assert out.returncode == 0, out.stderr[-2000:]
    assert [tuple(map(int, x.split())) for x in out.stdout.split("\n")[:-1]] == want
