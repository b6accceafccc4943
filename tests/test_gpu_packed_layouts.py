"""Layouts that the headers allow beside rows of packed heads: heads before tokens, tokens so far apart that offsets pass 32 bits, statistics that nobody
asks for, offsets of the keys given though they are the queries'.  The results are the bits of packed rows."""
import pytest

pytestmark = pytest.mark.gpu


def spread(x, st, sh):
    """A copy of [T, heads, D] with these strides."""
    import torch
    T, heads, D = x.shape
    y = torch.empty((T - 1) * st + (heads - 1) * sh + D, dtype=x.dtype, device=x.device).as_strided((T, heads, D), (st, sh, 1))
    y.copy_(x)
    return y


@pytest.mark.parametrize("D,layout", [(128, "heads_first"), (64, "heads_first"), (128, "far"), (64, "far"), (72, "heads_first"), (40, "far")])
def test_packed(D, layout):
    import torch
    from paper_2301_08984_amd import packed_binding as pb
    from packed_cases import Packed
    print(f"packed layout {D} {layout}", flush=True)
    lens, H, HK = [150, 0, 210], 6, 2
    T = sum(lens)
    a = Packed(91, lens, H, HK, D)
    a.fwd()
    a.bwd(True)
    strides = lambda heads: (D, T * D + 8) if layout == "heads_first" else ((1 << 23) + 8, D + 8)  # noqa: E731  (360 tokens: 6 GB)
    d = pb.make_desc(T, 3, H, HK, D, 0, HK, 1, **{f"{n}_stride_{w}": s for n, heads in (("q", H), ("k", HK), ("y", H)) for w, s in zip("th", strides(heads))})
    Q, K, V, dY = (spread(x, *strides(x.shape[1])) for x in (a.Q, a.K, a.V, a.dY))
    Y, dQ, dK, dV = (spread(torch.full_like(x, float("nan")), *strides(x.shape[1])) for x in (a.Y, a.dQ, a.dK, a.dV))
    st = torch.cuda.current_stream().cuda_stream
    pb.ss_packed_fwd(d, Q, K, V, a.dev_q, a.dev_q, Y, None, None, 0, st)
    for lse in (a.lse, None):
        for x in (dQ, dK, dV):
            x.fill_(float("nan"))
        pb.ss_packed_bwd(d, Q, K, V, a.dev_q, a.dev_q, None if lse is None else Y, dY, lse, dQ, dK, dV, a.ws, a.ws.numel(), st)
        a.bwd(lse is not None)
        torch.cuda.synchronize()
        for got, want in ((Y, a.Y), (dQ, a.dQ), (dK, a.dK), (dV, a.dV)):
            assert torch.equal(got, want)


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("H,new", [(4, [1, 1]), (16, [9, 3]), (8, [40, 1])], ids=["a_row", "72_rows", "160_rows"])
@pytest.mark.parametrize("layout", ["heads_first", "far"])
def test_cache(fmt, H, new, layout):
    import torch
    from cache_cases import Cache
    from paper_2301_08984_amd import cache_binding as cb
    print(f"cache layout {fmt} {H} {layout}", flush=True)
    a, b = (Cache(93, [700, 30], new, H, 2, 128, fmt, 16) for _ in range(2))
    T, D = sum(new), 128
    strides = (D, T * D + 8) if layout == "heads_first" else ((1 << 29) + 8, D + 8)
    if layout == "far" and T > 12:
        strides = ((1 << 27) + 8, D + 8)
    for c in (a, b):
        c.write("past")
    a.write("new")
    a.attn()
    K, V, Q = (spread(x, *strides) for x in (*b.kv["new"], b.Q))
    st = b.stream()
    cb.ss_cache_write(b.desc, T, K, V, *strides, b.cu["new"], b.start, b.dev_table, *b.store, st)
    for x, y in zip(a.store, b.store):
        if x is not None:
            assert torch.equal(torch.nan_to_num(x.float(), nan=-9.0), torch.nan_to_num(y.float(), nan=-9.0))
    Y = spread(torch.full_like(a.Y, float("nan")), *strides)
    d = cb.make_attn_desc(T, H, b.max_new, D, scale=b.scale, q_stride_t=strides[0], q_stride_h=strides[1], y_stride_t=strides[0], y_stride_h=strides[1])
    cb.ss_cache_attn(b.desc, d, Q, b.cu["new"], b.dev_lens, None, b.dev_table, *b.store, Y, None, b.ws, b.ws.numel(), st)
    back = [spread(torch.full_like(x, float("nan")), *strides) for x in b.kv["new"]]
    cb.ss_cache_read(b.desc, T, b.cu["new"], b.start, b.dev_table, *b.store, *back, *strides, st)
    want = a.read(T, a.cu["new"], a.start)
    torch.cuda.synchronize()
    assert torch.equal(Y, a.Y)
    for x, y in zip(back, want):
        assert torch.equal(x, y)
