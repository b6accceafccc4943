"""The kernels over the cache that keep keys and values in registers: nothing is spilled to memory and no accumulation register is in use, in any
format and head size (e4m3 at 128 takes nearly all of 256 registers)."""
import os
import subprocess

from paper_2301_08984_amd import build as B


def test_generated_code(tmp_path):
    out, src = str(tmp_path / "k.s"), "cache_attn.hip"
    r = subprocess.run(["hipcc", *B.FLAGS, *B.EXTRA_FLAGS[src], "--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = open(out).read().splitlines()
    assert not any("v_accvgpr" in x for x in lines)
    for what in (".agpr_count:", ".vgpr_spill_count:", ".private_segment_fixed_size:"):
        found = [x for x in lines if what in x]
        assert len(found) >= 10 and all(x.split()[-1] == "0" for x in found), what
