"""Packed attention's backward in several chunks of key heads one after the other, as it runs where the caller's workspace holds one chunk and
the library's buffer is not to be had (a call that is being captured): every number of chunks gives one chunk's bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

# lens_q, lens_k, H, HK, D, share, k; `parts`: the rows of dK and dV are cut into parts too
CASES = {
    "two": ([150, 64, 99], None, 12, 6, 64, (0, 6), 2),
    "uneven_three": ([150, 64, 99], None, 21, 7, 128, (0, 7), 3),
    "uneven_four_of_five": ([140, 300], None, 14, 7, 128, (1, 6), 4),
    "a_head_each": ([77, 0, 131], [200, 30, 131], 10, 5, 64, (0, 5), 5),
    "odd_head": ([333], None, 8, 4, 72, (1, 4), 3),
    "parts": ([900, 40], None, 24, 4, 128, (0, 4), 2),
    "parts_of_a_share": ([700], [900], 40, 5, 64, (2, 5), 3),
    "eight_parts": ([1300], None, 16, 2, 128, (0, 2), 2),
}


def chunks_that_run(c, keep):
    """How many chunks a call with `c`'s workspace and no other runs: the fewest of 1, 2, 4, .. whose scratch it holds (LSE and Delta of the
    largest chunk's query heads, only the latter with kept statistics, and what the parts' sums take)."""
    import copy
    k = 1
    while k < c.k:
        d = copy.copy(c.desc)
        d.k = k
        most = -(-(c.hi - c.lo) // k)
        stat = -(-most * (c.H // c.HK) * d.Tq * 4 // 256) * 256
        if c.pb.ss_packed_workspace_bytes(d)[1] - (stat if keep else 0) <= c.ws.numel():
            return k
        k *= 2
    return c.k


@pytest.mark.parametrize("keep", [False, True], ids=["recomputed", "kept"])
@pytest.mark.parametrize("name", CASES)
def test_captured_in_chunks(name, keep):
    import torch
    from packed_cases import Packed
    lens_q, lens_k, H, HK, D, share, k = CASES[name]
    print(f"packed chunks {name} keep={keep}", flush=True)
    one, c = (Packed(71, lens_q, H, HK, D, lens_k, before=3, behind=5, share=share, k=x) for x in (1, k))
    assert chunks_that_run(one, keep) == 1
    # (kept: half of the scratch, so that the workspace holds twice the heads)
    assert chunks_that_run(c, keep) > 1 or (keep and name in ("two", "uneven_three"))
    for x in (one, c):
        x.fwd()
    one.bwd(keep)
    torch.cuda.synchronize()
    one.check(one.oracle())
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        c.bwd(keep)
    for _ in range(3):
        for n in ("dQ", "dK", "dV"):
            getattr(c, n).fill_(float("nan"))
        c.ws.fill_(0xFF)
        one.bwd(not keep)
        graph.replay()
        torch.cuda.synchronize()
        one.bwd(keep)
        torch.cuda.synchronize()
        for n in ("dQ", "dK", "dV"):
            assert torch.equal(torch.nan_to_num(getattr(c, n), nan=7e7), torch.nan_to_num(getattr(one, n), nan=7e7)), n


def test_chunks_on_two_streams():
    """Two streams at once, of which at most one has the library's buffer at a time; the bits are one chunk's."""
    import torch
    from packed_cases import Packed
    print("packed chunks streams", flush=True)
    args = (73, [400, 90], 24, 8, 128)
    a, b, e = (Packed(*args, k=x) for x in (8, 3, 1))
    e.fwd()
    e.bwd(True)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(6):
        for c, st in ((a, torch.cuda.current_stream()), (b, side)):
            with torch.cuda.stream(st):
                c.fwd()
                c.bwd(i % 2 == 0)
    for c, st in ((a, torch.cuda.current_stream()), (b, side)):
        with torch.cuda.stream(st):
            c.bwd(True)
    torch.cuda.synchronize()
    for c in (a, b):
        for n in ("Y", "lse", "dQ", "dK", "dV"):
            assert torch.equal(getattr(c, n), getattr(e, n)), n
