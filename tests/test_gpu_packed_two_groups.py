"""Packed attention where two groups of wavefronts share a tile of rows (few tiles, sequences of 400 keys and more in the mean): lengths at the edges of
tiles and blocks beside long ones, empty sequences, more and fewer keys than queries, odd head sizes and groups."""
import pytest

pytestmark = pytest.mark.gpu

# lens_q, lens_k (None: the same), H, HK, D
CASES = {
    "edges": ([2800, 31, 33, 0, 64, 129, 1], None, 2, 1, 128),
    "edges64": ([2400, 127, 128, 65, 0, 32], None, 3, 1, 64),
    "few_blocks": ([500], None, 5, 5, 128),
    "few_blocks64": ([449], None, 4, 2, 64),
    "more_keys": ([5, 64, 1, 130], [70, 1500, 300, 257], 4, 2, 128),
    "more_keys64": ([1, 33, 100], [1000, 640, 449], 8, 2, 64),
    "fewer_keys": ([40, 900, 70], [7, 1300, 0], 3, 1, 128),
    "fewer_keys64": ([1200, 40], [800, 39], 4, 2, 64),
    "odd_head40": ([900], None, 4, 1, 40),
    "odd_head72": ([411, 700], None, 6, 2, 72),
    "odd_head96": ([70, 800, 400], None, 4, 2, 96),
    "many_tiles": ([1100], None, 32, 8, 128),
    "many_tiles64": ([1000], None, 32, 8, 64),
}


@pytest.mark.parametrize("keep", [True, False], ids=["kept", "recomputed"])
@pytest.mark.parametrize("name", CASES)
def test_against_the_oracle(name, keep):
    import torch
    from packed_cases import Packed
    lens_q, lens_k, H, HK, D = CASES[name]
    T = sum(lens_q) + 8
    tiles, keys = (T * (H // HK) >> 7) * HK, (sum(lens_k or lens_q) + 8) // len(lens_q)
    assert keys >= 400 if tiles < 256 else tiles <= 512 and keys >= 3 * tiles
    print(f"packed two groups {name} keep={keep}", flush=True)
    c = Packed(len(name), lens_q, H, HK, D, lens_k, before=3, behind=5)
    c.fwd()
    c.bwd(keep)
    torch.cuda.synchronize()
    c.check(c.oracle())
