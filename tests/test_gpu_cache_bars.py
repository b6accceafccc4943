"""Attention over the cache in 8 bits by the bars that its arithmetic has.  Codes become bf16 exactly (e4m3 has four significant bits, an int8 code seven; the
offset that an int8 conversion goes by is taken off before the product, exactly), so that scores are fp32 sums of exact products, times the scale, and
nothing but P (times V's scale) and the result is rounded to bf16."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

CASES = {  # past, new, H, HK, D, page
    "rows_in_registers": ([600, 5, 0, 1300, 90, 513], [3, 1, 2, 4, 0, 1], 8, 2, 128, 16),
    "rows_in_registers64": ([1, 800, 333], [1, 1, 2], 4, 2, 64, 8),
    "rows_that_share_tiles": ([600, 5, 900, 300], [40, 3, 64, 33], 8, 2, 128, 16),
    "up_to_64_rows64": ([800, 20, 450], [15, 16, 9], 12, 3, 64, 32),
}


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
@pytest.mark.parametrize("name", CASES)
def test_rounding_of_probabilities_and_results_alone(name, fmt):
    import torch
    from cache_cases import Cache
    from oracle import cache as oc
    from oracle import packed as op
    past, new, H, HK, D, page = CASES[name]
    print(f"cache bars {name} {fmt}", flush=True)
    c = Cache(101 + len(name), past, new, H, HK, D, fmt, page)
    c.write("past")
    c.write("new")
    c.attn()
    torch.cuda.synchronize()
    ref = oc.attention(c.Q.float().cpu().numpy(), *c.want_values(), c.table, page, c.cu["new"].cpu().numpy(), c.lens, None, c.scale, c.max_new)
    got, want = c.Y.float().cpu().numpy().astype(np.float64), ref["Y"]
    assert not np.isnan(got).any()
    # half a step of P against the magnitudes, half a step of the result; a sixteenth more for all that is fp32
    assert np.all(np.abs(got - want) <= op.bounds(ref, "Y") + 1e-30)
    # Both roundings are spread evenly over half a step (variance U^2 / 3 of the square), and with values of no mean the variance of sum P v is that of
    # the result itself: sqrt(2 / 3) U of its 2-norm, and a fifth more for chance
    assert np.linalg.norm(got - want) <= op.U * np.linalg.norm(want)
    lse = c.lse.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(lse - ref["lse"]) <= 2.0 ** -20 * (1 + np.abs(ref["lse"]) + ref["near"]))
