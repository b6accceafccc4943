"""The kernel of packed attention's Delta reads LDS from hand-written assembly, as its neighbours do (test_packed_isa.py): nothing touches a register
between a read and its wait, no accumulation register is in use, and nothing is spilled."""
import os
import subprocess

from paper_2301_08984_amd import build as B
from test_wave_isa import pending_read_violations


def test_generated_code(tmp_path):
    out, src = str(tmp_path / "k.s"), "packed_delta.hip"
    r = subprocess.run(["hipcc", *B.FLAGS, *B.EXTRA_FLAGS[src], "--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = open(out).read().splitlines()
    assert any("ds_read_b128" in x for x in lines)
    assert pending_read_violations(lines) == []
    assert not any("v_accvgpr" in x for x in lines)
    for what in (".agpr_count:", ".vgpr_spill_count:"):
        found = [x for x in lines if what in x]
        assert found and all(x.split()[-1] == "0" for x in found), what
