"""Delta of packed attention's backward where its error counts: dQ_i = scale sum_j P_ij (dP_ij - Delta_i) k_j, so an error e of Delta_i is
-scale e sum_j P_ij k_j in dQ_i, which the rest of the sum does not hide where the keys have a mean, or where one key has nearly all of a
row's probability (dS is then small, and its key is not).  Results go by a bar without any rounding of Delta to 16 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -8  # half a step of bf16, relative


def plain(c):
    """dQ, dK in 64 bits, and the 2-norm that their errors may have: dS and the result are rounded to bf16, each by at most half a step
    and evenly within it (variance U^2 / 3 of the value squared; a quarter more for chance); dP, Delta and P are 32-bit sums of D products and
    carry 2^-23 of a sum's magnitudes for each, and 2^-19 of P (its exponent has up to five digits before the point), all with one sign."""
    Q, K, V, dY = (c.host(n) for n in ("Q", "K", "V", "dY"))
    G, D = c.H // c.HK, c.D
    want = {"dQ": np.zeros_like(Q), "dK": np.zeros_like(K)}
    var, worst = ({n: np.zeros_like(x) for n, x in want.items()} for _ in range(2))
    for a, b, ka, kb in zip(c.cu_q[:-1], c.cu_q[1:], c.cu_k[:-1], c.cu_k[1:]):
        n, m = b - a, kb - ka
        seen = np.arange(m)[None, :] <= np.arange(n)[:, None] + (m - n)
        for h in range(c.H):
            q, k, v, g = Q[a:b, h], K[ka:kb, h // G], V[ka:kb, h // G], dY[a:b, h]
            s = np.where(seen, q @ k.T * c.scale, -np.inf)
            P = np.exp(s - s.max(1, keepdims=True))
            P /= P.sum(1, keepdims=True)
            dP, e = g @ v.T, D * 2.0 ** -23 * (abs(g) @ abs(v).T)
            dS = P * (dP - (P * dP).sum(1, keepdims=True))
            err = P * (e + (P * e).sum(1, keepdims=True)) + 2.0 ** -19 * abs(dS)
            want["dQ"][a:b, h] = c.scale * dS @ k
            want["dK"][ka:kb, h // G] += c.scale * dS.T @ q
            var["dQ"][a:b, h] = c.scale ** 2 * (dS ** 2 @ k ** 2)
            var["dK"][ka:kb, h // G] += c.scale ** 2 * (dS.T ** 2 @ q ** 2)
            worst["dQ"][a:b, h] = abs(c.scale) * err @ abs(k)
            worst["dK"][ka:kb, h // G] += abs(c.scale) * err.T @ abs(q)
    bar = {n: 1.25 * U * np.sqrt(np.sum(var[n] + want[n] ** 2) / 3) + np.linalg.norm(worst[n]) for n in want}
    return want, bar


@pytest.mark.parametrize("keep", [True, False], ids=["kept", "recomputed"])
@pytest.mark.parametrize("D,H,HK,lens_q,lens_k", [
    (128, 6, 2, [512, 90], None), (64, 8, 2, [512, 90], None), (128, 4, 2, [300, 40], [700, 500]), (72, 32, 16, [150] * 30, None),
], ids=["heads_of_128", "heads_of_64", "more_keys", "many_tiles"])
@pytest.mark.parametrize("data", ["means", "large_values", "one_key"])
def test_gradients_do_not_have_an_error_of_delta(data, D, H, HK, lens_q, lens_k, keep):
    import torch
    from packed_cases import Packed
    print(f"packed delta {data} {D} {H} {HK} keep={keep}", flush=True)
    c = Packed(61, lens_q, H, HK, D, lens_k)
    rng = np.random.default_rng(62)
    if data == "one_key":  # the first key of a sequence has most of every row's probability
        at = torch.from_numpy(c.cu_k[:-1].astype(np.int64)).cuda()
        c.Q[..., 0] = 8.0
        c.K[..., 0] = 0.0
        c.K[at, :, 0] = float(np.sqrt(D)) * 1.5
        c.V[at] *= 4.0
    else:  # one channel in twenty has a mean, in K and in V
        some = torch.from_numpy(rng.choice(D, D // 20, replace=False)).cuda()
        c.K[..., some] += 4.0
        c.V[..., some] += 4.0 if data == "means" else 16.0
    c.fwd()
    c.bwd(keep)
    torch.cuda.synchronize()
    want, bar = plain(c)
    for n in ("dQ", "dK"):
        off = float(np.linalg.norm(c.host(n) - want[n]))
        size = float(np.linalg.norm(want[n]))
        print(f"  {n}: {off / size:.5f} of its size, may be {bar[n] / size:.5f}", flush=True)
    for n in ("dQ", "dK"):
        assert np.linalg.norm(c.host(n) - want[n]) <= bar[n], n
