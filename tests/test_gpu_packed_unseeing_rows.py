"""Queries that see no key (a sequence with fewer keys than queries) pass no gradient on, whatever stands in their rows of Q and dY: the other
gradients are the bits that zeros there give, and their own dQ is 0."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("keep", [True, False], ids=["kept", "recomputed"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("lens_q,lens_k,H,HK,D", [
    ([40, 100, 70, 3], [7, 37, 0, 3], 4, 2, 128), ([40, 100, 70, 3], [7, 37, 0, 3], 6, 2, 64), ([300], [129], 5, 1, 128), ([900, 40], [640, 30], 16, 2, 72),
    ([50] * 70, [20] * 70, 32, 8, 128),
], ids=["several", "several64", "one", "parts", "many"])
def test_rows_without_a_key(lens_q, lens_k, H, HK, D, value, keep):
    import torch
    from packed_cases import Packed
    print(f"packed unseeing {lens_q[:4]} {D} {value} keep={keep}", flush=True)
    a, b = (Packed(81, lens_q, H, HK, D, lens_k, before=2, behind=3) for _ in range(2))
    rows = np.concatenate([np.arange(q, q + max(n - m, 0)) for q, n, m in zip(a.cu_q[:-1], lens_q, lens_k)])
    rows = torch.from_numpy(rows).cuda()
    a.Q[rows], a.dY[rows] = 0.0, 0.0
    b.Q[rows], b.dY[rows] = value, value
    for c in (a, b):
        c.fwd()
        c.bwd(keep)
    torch.cuda.synchronize()
    for c in (a, b):
        assert bool((c.Y[rows] == 0).all()) and bool((c.lse[:, rows] == float("-inf")).all()) and bool((c.dQ[rows] == 0).all())
    for n in ("Y", "lse", "dQ", "dK", "dV"):
        assert torch.equal(torch.nan_to_num(getattr(a, n), nan=7e7), torch.nan_to_num(getattr(b, n), nan=7e7)), n
