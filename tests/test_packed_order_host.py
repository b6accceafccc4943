"""The order in which the work-groups of packed attention take tiles, as numpy arithmetic: every (tile, head) is taken once, whatever
the number of heads, and the closed form of the number of tiles with at least L steps counts what it says."""
import numpy as np
import pytest


def place(block, HK):
    x, idx = block & 7, block >> 3
    q, a = idx // HK, HK >> 3
    rem = idx - q * HK
    if rem < 8 * a:
        return 8 * q + rem // a, x * a + rem % a
    rem -= 8 * a
    first = 8 * a
    if HK & 4:
        if rem < 4:
            return 8 * q + 2 * rem + (x & 1), first + (x >> 1)
        rem -= 4
        first += 4
    if HK & 2:
        if rem < 2:
            return 8 * q + 4 * rem + (x & 3), first + (x >> 2)
        first += 2
    return 8 * q + x, first


@pytest.mark.parametrize("HK", list(range(1, 26)) + [40, 96])
def test_every_tile_is_taken_once(HK):
    tiles = 43
    blocks = (tiles + 7) // 8 * 8 * HK
    seen = sorted(place(b, HK) for b in range(blocks))
    assert seen == [(r, h) for r in range((tiles + 7) // 8 * 8) for h in range(HK)]


def at_least(n, m, G, L, keys):
    more = m - n
    tiles = -(-(m if keys else n * G) // 128)
    if L <= 0:
        return tiles
    if keys:
        z = n - 1 - (32 * (L - 1)) // G
        return 0 if z < 0 or z + more < 0 else min(tiles, ((z + more) >> 7) + 1)
    y = 64 * (L - 1) - more
    return 0 if y >= n else tiles - ((max(y, 0) * G) >> 7)


@pytest.mark.parametrize("G", [1, 2, 3, 5, 8, 40])
def test_steps_of_tiles(G):
    rng = np.random.default_rng(G)
    for _ in range(300):
        n, m = int(rng.integers(0, 700)), int(rng.integers(0, 900))
        more, rows = m - n, n * G
        row_steps = [-(-max(min(128 * t + 127, rows - 1) // G + more + 1, 0) // 64) for t in range(-(-rows // 128))]
        assert row_steps == sorted(row_steps)  # the last tile is the heaviest
        key_rows = [(n - max(128 * t - more, 0)) * G for t in range(-(-m // 128))]
        key_steps = [-(-x // 32) if x > 0 else 0 for x in key_rows]
        for L in range(0, 20):
            assert at_least(n, m, G, L, False) == sum(x >= L for x in row_steps), (n, m, L)
            assert at_least(n, m, G, L, True) == sum(x >= L for x in key_steps), (n, m, L)
