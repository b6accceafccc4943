"""Pins of the fp64 oracles of packed attention and of the cache: brute force, finite differences, the dense oracle of the
framework's own attention, and the formats' definitions against torch's conversions."""
import math

import numpy as np
import pytest

from oracle import attention as dense
from oracle import cache as oc
from oracle import packed as op


def _case(seed, lens_q, lens_k, H, HK, D):
    rng = np.random.default_rng(seed)
    cu_q, cu_k = (np.concatenate([[0], np.cumsum(x)]) for x in (lens_q, lens_k))
    Q, dY = rng.normal(size=(2, cu_q[-1], H, D))
    K, V = rng.normal(size=(2, cu_k[-1], HK, D))
    return Q, K, V, dY, cu_q, cu_k


def test_against_loops():
    Q, K, V, dY, cu_q, cu_k = _case(1, [3, 0, 1, 4], [5, 2, 1, 2], 4, 2, 8)
    out = op.attention(Q, K, V, cu_q, cu_k, 0.3, dY)
    for b in range(4):
        n, m = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        for h in range(4):
            for i in range(n):
                t = cu_q[b] + i
                keys = [j for j in range(m) if j <= i + m - n]
                w = [math.exp(0.3 * sum(Q[t, h, d] * K[cu_k[b] + j, h // 2, d] for d in range(8))) for j in keys]
                want = sum((x * V[cu_k[b] + j, h // 2] for x, j in zip(w, keys)), np.zeros(8)) / (sum(w) or 1.0)
                np.testing.assert_allclose(out["Y"][t, h], want, atol=1e-12)
                assert out["lse"][h, t] == (pytest.approx(math.log(sum(w))) if keys else -math.inf)
    assert np.all(out["Y"][cu_q[3]:cu_q[3] + 2] == 0) and np.all(out["dQ"][cu_q[3]:cu_q[3] + 2] == 0)  # queries that see no key
    assert np.all(out["dK"][cu_k[1]:cu_k[2]] == 0)                                                     # keys that no query sees


def test_gradients_against_differences():
    Q, K, V, dY, cu_q, cu_k = _case(2, [4, 3], [4, 6], 2, 1, 8)
    out = op.attention(Q, K, V, cu_q, cu_k, 0.4, dY)
    rng, h = np.random.default_rng(3), 1e-5
    for name, x in (("dQ", Q), ("dK", K), ("dV", V)):
        for _ in range(12):
            i = tuple(rng.integers(0, s) for s in x.shape)
            keep, f = x[i], []
            for d in (h, -h):
                x[i] = keep + d
                f.append(float((op.attention(Q, K, V, cu_q, cu_k, 0.4)["Y"] * dY).sum()))
            x[i] = keep
            assert out[name][i] == pytest.approx((f[0] - f[1]) / (2 * h), rel=1e-6, abs=1e-8), name


def test_one_sequence_is_the_dense_operator():
    Q, K, V, dY, cu, _ = _case(4, [9], [9], 3, 3, 16)
    out = op.attention(Q, K, V, cu, cu, 0.25, dY)
    p = dense.AttnProblem(Q[None], K[None], V[None], 0.25, None, ("causal",), None)
    Y, lse = dense.attn_forward(p, dense.AXIS_HEAD, 0, 3)
    g = dense.attn_backward(p, dY[None], dense.AXIS_HEAD, 0, 3)
    np.testing.assert_allclose(out["Y"], Y[0], atol=1e-12)
    np.testing.assert_allclose(out["lse"], lse[0], atol=1e-12)
    for n in ("dQ", "dK", "dV"):
        np.testing.assert_allclose(out[n], g[n][0], atol=1e-12)


def test_formats():
    import torch
    assert len(oc._E4M3) == 127 and oc._E4M3[-1] == 448.0
    np.testing.assert_array_equal(oc._E4M3, torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())
    rng = np.random.default_rng(5)
    x = torch.from_numpy(rng.normal(size=(400, 64)) * np.exp(rng.uniform(-80, 80, size=(400, 1)))).to(torch.bfloat16).float().numpy()
    x[3], x[4, 1:] = 0.0, 0.0
    codes, scale = oc.quantise(x, oc.FP8)
    want = (torch.from_numpy(x) / torch.from_numpy(scale.astype(np.float32))[:, None]).to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(codes, want)
    most = np.abs(x).max(1)
    live = most > 448 * 2.0 ** -126
    assert np.all(most[live] <= 448 * scale[live]) and np.all(most[live] > 224 * scale[live])
    codes, scale = oc.quantise(x, oc.INT8)
    assert np.abs(codes).max() == 127 and np.all(codes == np.rint(codes))
    assert np.all(np.abs(codes * scale[:, None] - x) <= 0.5001 * scale[:, None])
    x[7, 2], x[8, 0] = np.nan, -np.inf
    for fmt in (oc.FP8, oc.INT8):
        assert np.isnan(oc.quantise(x, fmt)[1][7:9]).all() and np.isfinite(oc.quantise(x, fmt)[0]).all()


def test_the_bounds_notice_a_planted_mistake():
    """A key left out, a head taken from the wrong group: outside the 2-norm bar that the kernels are held to."""
    from packed_cases import off
    Q, K, V, dY, cu, _ = _case(6, [200], [200], 4, 2, 16)
    out = op.attention(Q, K, V, cu, cu, 0.25, dY)
    K2 = K.copy()
    K2[100] = -1e3
    wrong = op.attention(Q, K2, V, cu, cu, 0.25, dY)
    assert off(wrong["Y"], out["Y"]) > 2 * op.U
    wrong = op.attention(Q, K[:, ::-1], V, cu, cu, 0.25, dY)
    assert all(off(wrong[n], out[n]) > 3 * op.U for n in ("Y", "dQ", "dK", "dV"))
