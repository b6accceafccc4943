"""The kernels of packed attention, and of many rows over the cache, read LDS from hand-written assembly: nothing touches a register between a read and its
wait, no accumulation register is in use, and nothing is spilled (test_wave_isa.py, whose checks these are)."""
import os
import subprocess

import pytest

from paper_2301_08984_amd import build as B
from test_wave_isa import pending_read_violations


@pytest.mark.parametrize("src", ["packed_fwd.hip", "packed_dq.hip", "packed_dkdv.hip", "cache_attn_rows.hip"])
def test_generated_code(src, tmp_path):
    out = str(tmp_path / "k.s")
    r = subprocess.run(["hipcc", *B.FLAGS, *B.EXTRA_FLAGS[src], "--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = open(out).read().splitlines()
    assert any("ds_read_b64_tr_b16" in x for x in lines)
    assert pending_read_violations(lines) == []
    assert not any("v_accvgpr" in x for x in lines)
    for what in (".agpr_count:", ".vgpr_spill_count:"):
        found = [x for x in lines if what in x]
        assert found and all(x.split()[-1] == "0" for x in found), what
