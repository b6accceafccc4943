"""Offsets of the cache's packed tokens that lie outside 0 .. T are clamped: the first row that is left has the position `start` names."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first,last", [(-3, 14), (0, 2 ** 31 - 1), (-2 ** 31, 2 ** 31 - 1)])
@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
def test_offsets_outside_the_tokens(fmt, first, last):
    import torch
    from cache_cases import Cache
    print(f"cache offsets {fmt} {first} {last}", flush=True)
    a, b = (Cache(7, [20, 37], [6, 8], 4, 2, 64, fmt, 16) for _ in range(2))
    b.cu["new"][0], b.cu["new"][2] = first, last
    out = []
    for c in (a, b):
        c.write("past")
        c.write("new")
        c.attn()
        out.append([*c.read(14, c.cu["new"], c.start), c.Y, c.lse])
    torch.cuda.synchronize()
    for x, y in zip(a.store, b.store):
        if x is not None:
            assert torch.equal(torch.nan_to_num(x.float(), nan=-9.0), torch.nan_to_num(y.float(), nan=-9.0))
    for x, y in zip(*out):
        assert not torch.isnan(x).any() and torch.equal(x, y)
