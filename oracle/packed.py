"""Attention over packed sequences with grouped heads, plainly, in fp64 numpy: one sequence and one query head at a
time.  Beside the results `attention` gives, for every result, the sums of magnitudes that bound what a kernel's
roundings to bf16 can do to it (see `bounds`)."""
import numpy as np

U = 2.0 ** -8  # half a step of bf16, relative


def sequences(cu_q, cu_k):
    """(first query, queries, first key, keys) of every sequence."""
    return [(int(cu_q[b]), int(cu_q[b + 1] - cu_q[b]), int(cu_k[b]), int(cu_k[b + 1] - cu_k[b])) for b in range(len(cu_q) - 1)]


def head(q, k, v, scale, dy=None, see=None):
    """One query head of one sequence: q [n,D], k, v [m,D]; `see` [n,m]: visible pairs (None: causal, the queries being the last)."""
    n, m = len(q), len(k)
    if see is None:
        see = np.arange(m)[None, :] <= np.arange(n)[:, None] + (m - n)
    s = np.where(see, scale * (q @ k.T), -np.inf)
    top = s.max(1, initial=-np.inf, keepdims=True)
    e = np.where(see, np.exp(s - np.where(np.isfinite(top), top, 0.0)), 0.0)
    total = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(total))[:, 0]
    p = e / np.where(total == 0, 1.0, total)
    r = {"Y": p @ v, "lse": lse, "P": p, "near": abs(scale) * (np.abs(q) @ np.abs(k).T).max(1, initial=0.0)}
    r["Y_mag"] = p @ np.abs(v)
    if dy is not None:
        dp = dy @ v.T
        delta = (dy * r["Y"]).sum(1, keepdims=True)
        ds = p * (dp - delta)
        # what the rounding of P and of Y does to Delta
        off = U * (np.abs(dy) * (r["Y_mag"] + np.abs(r["Y"]))).sum(1, keepdims=True)
        ds_off = U * np.abs(ds) + p * off
        r.update(dQ=scale * ds @ k, dK=scale * ds.T @ q, dV=p.T @ dy)
        r.update(dQ_mag=abs(scale) * ds_off @ np.abs(k) / U, dK_mag=abs(scale) * ds_off.T @ np.abs(q) / U, dV_mag=p.T @ np.abs(dy))
    return r


def attention(Q, K, V, cu_q, cu_k, scale, dY=None):
    """Q, dY [Tq,H,D], K, V [Tk,HK,D] (any float type) -> dict of fp64 arrays: Y, lse [H,Tq], and with dY dQ, dK, dV; NaN in rows
    of no sequence.  NAME_mag: magnitudes for `bounds`."""
    Q, K, V = (np.asarray(x, np.float64) for x in (Q, K, V))
    (Tq, H, D), (Tk, HK, _) = Q.shape, K.shape
    out = {n: np.full((Tq, H, D), np.nan) for n in ("Y", "Y_mag")}
    out["lse"], out["near"] = np.full((H, Tq), np.nan), np.zeros((H, Tq))
    if dY is not None:
        dY = np.asarray(dY, np.float64)
        for n, T, heads in (("dQ", Tq, H), ("dK", Tk, HK), ("dV", Tk, HK)):
            out[n], out[n + "_mag"] = np.full((T, heads, D), np.nan), np.full((T, heads, D), np.nan)
    for a, n, c, m in sequences(cu_q, cu_k):
        if dY is not None:
            for name in ("dK", "dV", "dK_mag", "dV_mag"):
                out[name][c:c + m] = 0.0
        for h in range(H):
            g = h // (H // HK)
            r = head(Q[a:a + n, h], K[c:c + m, g], V[c:c + m, g], scale, None if dY is None else dY[a:a + n, h])
            for name in ("Y", "Y_mag") + (("dQ", "dQ_mag") if dY is not None else ()):
                out[name][a:a + n, h] = r[name]
            out["lse"][h, a:a + n], out["near"][h, a:a + n] = r["lse"], r["near"]
            if dY is not None:
                for name in ("dK", "dV", "dK_mag", "dV_mag"):
                    out[name][c:c + m, g] += r[name]
    return out


def bounds(out, name):
    """How far an element may be off: half a step of bf16 for the rounded operand of the last product (P or dS: times the
    sum of the products' magnitudes), and for the result itself; 1/16 more for everything that is held in fp32."""
    return 17.0 / 16.0 * U * (out[name + "_mag"] + np.abs(out[name]))
