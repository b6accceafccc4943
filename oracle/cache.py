"""The paged cache and the attention of new tokens over it, plainly: numpy, one row and one head at a time."""
import numpy as np

from . import packed

BF16, FP8, INT8 = 0, 1, 2
# the finite values of e4m3 from 0 on: 8 steps of 2^-9, then 8 a power of two
_E4M3 = np.array([i * 2.0 ** -9 for i in range(8)] + [(8 + i) * 2.0 ** (e - 10) for e in range(1, 16) for i in range(8)])[:127]


def quantise(x, fmt):
    """Rows [..., D] of fp32 values (bf16 numbers) -> (what the codes stand for without the scale, scales [...])."""
    x = np.asarray(x, np.float32)
    if fmt == BF16:
        return x.astype(np.float64), np.ones(x.shape[:-1])
    most = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    safe = np.where(bad | (most == 0), np.float32(1), most).astype(np.float32)
    if fmt == INT8:
        scale = np.maximum(safe / np.float32(127), np.float32(2.0 ** -126))
    else:
        scale = np.ones_like(safe)
        for i in np.ndindex(safe.shape):
            e = -126
            while float(safe[i]) > 448 * 2.0 ** e:
                e += 1
            scale[i] = 2.0 ** e
    scale = np.where(bad | (most == 0), np.float32(1), scale).astype(np.float32)
    quotient = np.where(bad[..., None], np.float32(0), x) / scale[..., None]  # fp32
    if fmt == INT8:
        codes = np.rint(quotient).astype(np.float64)
    else:
        a = np.abs(quotient).astype(np.float64)
        hi = np.clip(np.searchsorted(_E4M3, a), 0, 126)
        lo = np.maximum(hi - 1, 0)
        dh, dl = _E4M3[hi] - a, a - _E4M3[lo]
        take = np.where(dh < dl, hi, np.where(dl < dh, lo, np.where(lo % 2 == 0, lo, hi)))  # to even at a tie
        codes = np.where(a == _E4M3[hi], _E4M3[hi], _E4M3[take]) * np.sign(quotient)
    return codes, np.where(bad, np.nan, scale.astype(np.float64))


def values(x, fmt):
    codes, scale = quantise(x, fmt)
    return codes * scale[..., None]


def find(table, n_pages, page, b, pos):
    """(pool's page, slot) of a position, or None where there is none."""
    if pos < 0 or pos >= table.shape[1] * page:
        return None
    at = int(table[b, pos // page])
    return (at, pos % page) if 0 <= at < n_pages else None


def attention(Q, k_values, v_values, table, page, cu, lens, tree, scale, max_new):
    """Q [T,H,D]; k_values, v_values [n_pages,HK,page,D]: what the cache stands for -> Y, lse, magnitudes; NaN in rows that
    are not written."""
    Q = np.asarray(Q, np.float64)
    (T, H, D), (n_pages, HK) = Q.shape, k_values.shape[:2]
    out = {"Y": np.full((T, H, D), np.nan), "Y_mag": np.full((T, H, D), np.nan), "lse": np.full((H, T), np.nan), "near": np.zeros((H, T))}
    for b in range(len(cu) - 1):
        a, n = int(cu[b]), int(cu[b + 1] - cu[b])
        before, rows = max(int(lens[b]) - n, 0), min(n, max_new)
        places = [find(table, n_pages, page, b, j) for j in range(int(lens[b]))]
        there = [j for j, at in enumerate(places) if at is not None]
        see = np.zeros((rows, len(there)), bool)
        for i in range(rows):
            bits = (1 << (i + 1)) - 1 if tree is None else int(tree[a + i]) & (1 << 64) - 1
            see[i] = [j < before or (j - before < 64 and bool(bits >> (j - before) & 1)) for j in there]
        for h in range(H):
            g = h // (H // HK)
            k = np.array([k_values[places[j][0], g, places[j][1]] for j in there]).reshape(-1, D)
            v = np.array([v_values[places[j][0], g, places[j][1]] for j in there]).reshape(-1, D)
            with np.errstate(invalid="ignore"):
                r = packed.head(Q[a:a + rows, h], k, v, scale, see=see)
            out["Y"][a:a + rows, h], out["Y_mag"][a:a + rows, h] = r["Y"], r["Y_mag"]
            out["lse"][h, a:a + rows], out["near"][h, a:a + rows] = r["lse"], r["near"]
    return out
