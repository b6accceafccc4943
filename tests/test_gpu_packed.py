"""Attention over packed sequences with grouped heads against the fp64 oracle, through the C ABI."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

# lens_q, lens_k (None: the same), H, HK, D
CASES = {
    "one_token": ([1], None, 1, 1, 64),
    "single_tokens": ([1, 1, 1, 1, 1], None, 4, 2, 128),
    "with_empty": ([0, 5, 0, 33, 0, 0, 64, 0], None, 4, 4, 128),
    "edges": ([31, 32, 33, 63, 64, 65, 127, 128, 129], None, 6, 2, 128),
    "edges64": ([31, 32, 33, 63, 64, 65, 127, 128, 129], None, 8, 2, 64),
    "group_of_three": ([200, 7, 150], None, 3, 1, 128),
    "group_of_eight": ([130, 300], None, 8, 1, 128),
    "group_of_five": ([77, 140], None, 10, 2, 64),
    "many_heads": ([90, 41], None, 24, 12, 128),
    "five_key_heads": ([257], None, 5, 5, 64),
    "eleven_key_heads": ([140, 60], None, 11, 11, 128),
    "small_head": ([70, 65], None, 4, 2, 8),
    "odd_head40": ([70, 131], None, 4, 1, 40),
    "odd_head96": ([70, 131], None, 4, 2, 96),
    "odd_head120": ([65, 40], None, 2, 2, 120),
    "long": ([1100, 3, 700], None, 4, 2, 128),
    "long64": ([1025], None, 4, 4, 64),
    "more_keys": ([5, 64, 1, 130], [70, 64, 300, 257], 4, 2, 128),
    "more_keys64": ([1, 40], [1000, 40], 8, 2, 64),
    "fewer_keys": ([40, 100, 70, 3], [7, 37, 0, 3], 4, 2, 128),
    "no_queries": ([0, 20, 0], [30, 20, 129], 2, 1, 64),
    "many_sequences": ([3, 40, 0, 17] * 40, None, 4, 2, 64),
    "parts": ([900, 40], None, 12, 2, 128),
    "parts64": ([1100], [1300], 8, 1, 64),
    "parts_odd_head": ([700, 0, 300], None, 16, 2, 72),
    "eight_parts": ([1300], None, 8, 1, 128),
    "eight_parts64": ([1100, 2], [1100, 500], 24, 1, 64),
    "parts_without_queries": ([2000, 0, 30], [2000, 300, 30], 8, 1, 128),
    "short_rows": ([64] * 95 + [130, 1, 0, 300], None, 32, 16, 128),
    "short_and_long": ([100] * 50 + [400, 0, 700, 33, 129], None, 32, 4, 128),
    "short64": ([107] * 60 + [200, 3], None, 32, 8, 64),
    "short_five_key_heads": ([90] * 63 + [250], None, 35, 5, 96),
    "short_more_keys": ([40, 90, 10] * 50, [100, 90, 7] * 50, 32, 8, 128),
    "many_tiles": ([64] * 66 + [130], None, 32, 16, 128),
    "many_tiles64": ([70] * 60 + [131], None, 32, 16, 64),
    "some_tiles": ([64] * 66 + [130], None, 16, 8, 128),
    "some_tiles64": ([70] * 60 + [131], None, 16, 8, 64),
    "three_hundred_sequences": ([(7 * i) % 23 for i in range(300)], None, 2, 1, 128),
}


@pytest.mark.parametrize("keep", [True, False], ids=["kept", "recomputed"])
@pytest.mark.parametrize("name", CASES)
def test_against_the_oracle(name, keep):
    import torch
    from packed_cases import Packed
    lens_q, lens_k, H, HK, D = CASES[name]
    print(f"packed {name} keep={keep}", flush=True)
    c = Packed(len(name), lens_q, H, HK, D, lens_k, before=3, behind=5)
    c.fwd()
    c.bwd(keep)
    torch.cuda.synchronize()
    c.check(c.oracle())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("peaked,offset", [(6.0, 0.0), (1.0, 2.0), (0.0, 1.0)])
def test_peaked_offset_and_flat_data(D, peaked, offset):
    """Rows that one key decides; V and dY with a mean of their own; scores that are all the same."""
    import torch
    from packed_cases import Packed
    print(f"packed data {D} {peaked} {offset}", flush=True)
    c = Packed(17, [190, 260], 4, 2, D, peaked=peaked, offset=offset)
    c.fwd()
    c.bwd(True)
    torch.cuda.synchronize()
    c.check(c.oracle())


@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-3, 0.5])
def test_scales(scale):
    import torch
    from packed_cases import Packed
    print(f"packed scale {scale}", flush=True)
    c = Packed(19, [70, 140], 4, 2, 128, scale=scale)
    c.fwd()
    c.bwd(False)
    torch.cuda.synchronize()
    c.check(c.oracle())


def test_strides_and_share():
    """Rows with room between them, a range of key heads, and the same bits for every k."""
    import torch
    from packed_cases import Packed
    print("packed strides", flush=True)
    names = ("Y", "lse", "dQ", "dK", "dV")
    c = Packed(21, [150, 64, 99], 12, 6, 64, pad=8, before=2, behind=70, share=(1, 5))
    c.fwd()
    c.bwd(True)
    torch.cuda.synchronize()
    c.check(c.oracle())
    for k in (2, 3, 4):
        o = Packed(21, [150, 64, 99], 12, 6, 64, pad=8, before=2, behind=70, share=(1, 5), k=k)
        o.fwd()
        o.bwd(True)
        torch.cuda.synchronize()
        for n in names:
            assert torch.equal(torch.nan_to_num(getattr(o, n), nan=7e7), torch.nan_to_num(getattr(c, n), nan=7e7)), (k, n)


def test_slices_of_one_buffer():
    import torch
    from paper_2301_08984_amd import packed_binding as pb
    from packed_cases import Packed
    print("packed fused", flush=True)
    a = Packed(23, [100, 130], 6, 2, 128)
    a.fwd()
    a.bwd(True)
    T, H, HK, D = 230, 6, 2, 128
    qkv = torch.cat([a.Q, a.K, a.V], 1).contiguous()
    grads = torch.full_like(qkv, float("nan"))
    Y = torch.full((T, H, D), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    d = pb.make_desc(T, 2, H, HK, D, 0, HK, 1, q_stride_t=qkv.stride(0), k_stride_t=qkv.stride(0))
    cut = lambda x: (x[:, :H], x[:, H:H + HK], x[:, H + HK:])  # noqa: E731
    st = torch.cuda.current_stream().cuda_stream
    pb.ss_packed_fwd(d, *cut(qkv), a.dev_q, None, Y, a.lse, None, 0, st)
    pb.ss_packed_bwd(d, *cut(qkv), a.dev_q, None, Y, a.dY, a.lse, *cut(grads), a.ws, a.ws.numel(), st)
    torch.cuda.synchronize()
    assert torch.equal(Y, a.Y)
    for got, want in zip(cut(grads), (a.dQ, a.dK, a.dV)):
        assert torch.equal(got, want)


def test_garbage_outside_a_sequence_has_no_influence():
    """NaN and infinities in the other sequences: this one's rows are the same bits."""
    import torch
    from packed_cases import Packed
    print("packed garbage", flush=True)
    a, b = (Packed(25, [45, 100, 77], 4, 2, 128) for _ in range(2))
    for x in (b.Q, b.K, b.V, b.dY):
        x[:45] = float("nan")
        x[145:] = float("inf")
    for c in (a, b):
        c.fwd()
        c.bwd(False)
    torch.cuda.synchronize()
    for n in ("Y", "dQ", "dK", "dV"):
        assert torch.equal(getattr(a, n)[45:145], getattr(b, n)[45:145]), n
    assert torch.equal(a.lse[:, 45:145], b.lse[:, 45:145])


@pytest.mark.parametrize("cu", [[-5, 40, 300, 90], [100, 30, 60, 2 ** 31 - 1], [0, 0, 0, 0], [-2 ** 31, -1, 200, 1000]])
def test_wrong_offsets_stay_inside_the_tensors(cu):
    """Offsets that are out of range or fall: the calls end, and rows before the first and behind the last stay as they were.
    (The tensors lie between guard rows of the same allocation.)"""
    import torch
    from packed_cases import Packed
    print(f"packed offsets {cu}", flush=True)
    c = Packed(27, [60, 50, 40], 4, 2, 128)
    guard = {}
    for n in ("Y", "dQ", "dK", "dV"):
        x = getattr(c, n)
        full = torch.full((x.shape[0] + 512, *x.shape[1:]), 3.0, dtype=x.dtype, device=x.device)
        setattr(c, n, full[256:-256])
        guard[n] = full
    c.dev_q = torch.tensor(cu, dtype=torch.int32, device="cuda:0")
    c.fwd()
    c.bwd(False)
    torch.cuda.synchronize()
    for n, full in guard.items():
        assert bool((full[:256] == 3.0).all()) and bool((full[-256:] == 3.0).all()), n


def test_captured_and_replayed():
    """One graph of forward and backward over offsets that change between the replays."""
    import torch
    from packed_cases import Packed
    print("packed captured", flush=True)
    c = Packed(29, [150, 20, 130], 4, 2, 128)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        c.fwd()
        c.bwd(True)
    for lens in ([150, 20, 130], [1, 299, 0], [100, 100, 100], [150, 20, 130]):
        e = Packed(29, [150, 20, 130], 4, 2, 128)
        cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32)
        c.dev_q.copy_(cu)
        e.dev_q.copy_(cu)
        for n in ("Y", "dQ", "dK", "dV", "lse"):
            getattr(c, n).fill_(float("nan"))
        c.ws.fill_(0xFF)
        graph.replay()
        e.fwd()
        e.bwd(True)
        torch.cuda.synchronize()
        for n in ("Y", "lse", "dQ", "dK", "dV"):
            assert torch.equal(getattr(c, n), getattr(e, n)), (lens, n)


def test_two_streams():
    import torch
    from packed_cases import Packed
    print("packed streams", flush=True)
    a, b, e = (Packed(31, [400, 90], 8, 2, 128) for _ in range(3))
    e.fwd()
    e.bwd(True)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        for c, st in ((a, torch.cuda.current_stream()), (b, side)):
            with torch.cuda.stream(st):
                c.fwd()
                c.bwd(True)
    torch.cuda.synchronize()
    for c in (a, b):
        for n in ("Y", "lse", "dQ", "dK", "dV"):
            assert torch.equal(getattr(c, n), getattr(e, n)), n


@pytest.mark.parametrize("D,H,HK", [(64, 8, 2), (128, 6, 2), (128, 40, 8)])
def test_rows_of_few_keys_have_delta_from_products(D, H, HK):
    """V = 64 and a little: Y is off by up to a quarter there, and Delta = dY . Y with it by more than dS is large.  Rows of up to 64 keys do
    not go by it.  Their dS is off by P (the errors of dP and of Delta), which are fp32 sums of D products, and P's own 2^-19; then by half a step
    of bf16, as the result is."""
    import torch
    from packed_cases import Packed
    print(f"packed delta {D} {H} {HK}", flush=True)
    lens = [2, 3, 64, 1, 40, 9, 33, 64]
    c = Packed(29, lens, H, HK, D)
    rng = np.random.default_rng(30)
    c.V[:] = torch.from_numpy(64 + 0.5 * rng.integers(0, 9, size=tuple(c.V.shape))).cuda().bfloat16()
    c.fwd()
    c.bwd(True)
    torch.cuda.synchronize()
    Q, K, V, dY = (c.host(n) for n in ("Q", "K", "V", "dY"))
    G, half = H // HK, 2.0 ** -8
    want, bar = {n: np.zeros_like(x) for n, x in (("dQ", Q), ("dK", K))}, {}
    bar = {n: np.zeros_like(x) for n, x in want.items()}
    for a, b in zip(c.cu_q[:-1], c.cu_q[1:]):
        seen = np.tril(np.ones((b - a, b - a), bool))
        for h in range(H):
            q, k, v, g = Q[a:b, h], K[a:b, h // G], V[a:b, h // G], dY[a:b, h]
            s = np.where(seen, q @ k.T * c.scale, -np.inf)
            P = np.exp(s - s.max(1, keepdims=True))
            P /= P.sum(1, keepdims=True)
            dP, e = g @ v.T, D * 2.0 ** -23 * (abs(g) @ abs(v).T)
            dS = P * (dP - (P * dP).sum(1, keepdims=True))
            err = P * (e + (P * e).sum(1, keepdims=True) + 2.0 ** -19 * (P * abs(dP)).sum(1, keepdims=True)) + 2.0 ** -19 * abs(dS)
            err = half * abs(dS) + (1 + half) * err
            want["dQ"][a:b, h] = c.scale * dS @ k
            bar["dQ"][a:b, h] = c.scale * err @ abs(k)
            want["dK"][a:b, h // G] += c.scale * dS.T @ q
            bar["dK"][a:b, h // G] += c.scale * err.T @ abs(q)
    for n in ("dQ", "dK"):
        room = bar[n] * (1 + half) + half * abs(want[n]) + 1e-30
        assert np.all(abs(c.host(n) - want[n]) <= room), (n, float(np.max(abs(c.host(n) - want[n]) / room)))


def test_parts_captured_and_replayed():
    """dK and dV in eight parts: a captured call, replayed between eager work, gives the eager call's bits."""
    import torch
    from packed_cases import Packed
    print("packed parts captured", flush=True)
    a, b = (Packed(31, [1300], 8, 1, 128) for _ in range(2))
    for c in (a, b):
        c.fwd()
        c.bwd(True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.bwd(True)
    for _ in range(3):
        for x in (b.dQ, b.dK, b.dV):
            x.fill_(float("nan"))
        b.ws.fill_(0xFF)
        a.bwd(False)
        graph.replay()
        torch.cuda.synchronize()
        a.bwd(True)
        torch.cuda.synchronize()
        for n in ("dQ", "dK", "dV"):
            assert torch.equal(getattr(a, n), getattr(b, n)), n
