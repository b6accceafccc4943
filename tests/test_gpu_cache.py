"""The paged cache and the attention of new tokens over it against the oracle, through the C ABI."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("page,HK", [(8, 1), (16, 3), (64, 8), (1024, 5)])
def test_written_rows_read_back(fmt, page, HK, D):
    """Every value is the code's of the definition times its scale, rounded once, and nothing else changes."""
    import torch
    from cache_cases import Cache
    from oracle import cache as oc
    print(f"cache rows {fmt} {page} {HK} {D}", flush=True)
    c = Cache(page + HK, [30, 0, 1, 130], [5, 20, 0, 9], 2 * HK, HK, D, fmt, page)
    K = c.kv["new"][0]
    K[0, 0] = 0.0                                   # a row of zeros
    K[1, 0] = 1e-40                                 # subnormal
    K[2, 0, 1:] = 0.0                               # one value
    K[3, 0] *= 1e30
    K[4, 0] = torch.arange(-(D // 2), D // 2, device="cuda:0").bfloat16() / 4.0  # ties
    if fmt != "bf16":
        K[6, 0, 5] = float("nan")
        K[7, 0, 3] = float("-inf")
    c.write("past")
    before = [None if x is None else x.clone() for x in c.store]
    c.write("new")
    cu_all = torch.from_numpy(np.concatenate([[0], np.cumsum(c.lens)]).astype(np.int32)).cuda()
    T = int(cu_all[-1])
    got = [x.float().cpu().numpy() for x in c.read(T + 4, cu_all, None)]
    tail = [x.float().cpu().numpy() for x in c.read(K.shape[0], c.cu["new"], c.start)]
    torch.cuda.synchronize()
    at = at_new = at_past = 0
    for b, (p, n) in enumerate(zip(c.past, c.new)):
        for j in range(2):
            rows = np.concatenate([oc.values(c.host_kv("past")[j][at_past:at_past + p], c.fmt), oc.values(c.host_kv("new")[j][at_new:at_new + n], c.fmt)])
            with np.errstate(over="ignore"):
                rows = torch.from_numpy(rows).to(torch.bfloat16).float().numpy()
            np.testing.assert_array_equal(got[j][at:at + p + n], rows)
            np.testing.assert_array_equal(tail[j][at_new:at_new + n], rows[p:])
        at, at_new, at_past = at + p + n, at_new + n, at_past + p
    assert np.isnan(got[0][T:]).all()
    # the slots of the other tokens hold what they held
    slots = torch.zeros((c.n_pages, c.HK, page), dtype=torch.bool, device="cuda:0")
    for b in range(4):
        for pos in range(c.past[b], c.past[b] + c.new[b]):
            slots[int(c.table[b, pos // page]), :, pos % page] = True
    for old, now in zip(before, c.store):
        if old is not None:
            same = (old == now) | (torch.isnan(old) & torch.isnan(now)) if old.is_floating_point() else old == now
            assert bool(same.view(c.n_pages, c.HK, page, -1)[~slots].all())


def test_strided_rows():
    """K and V as slices of one projection's output, and read back into slices."""
    import torch
    from cache_cases import Cache
    print("cache strides", flush=True)
    a, b = (Cache(3, [40, 9], [6, 3], 4, 2, 64, "int8", 16) for _ in range(2))
    for c in (a, b):
        c.write("past")
    K, V = b.kv["new"]
    fused = torch.cat([K, K, V], 1).contiguous()
    b.cb.ss_cache_write(b.desc, 9, fused[:, 2:4], fused[:, 4:], fused.stride(0), 64, b.cu["new"], b.start, b.dev_table, *b.store, b.stream())
    a.write("new")
    for x, y in zip(a.store, b.store):
        assert torch.equal(torch.nan_to_num(x.float(), nan=-9.0), torch.nan_to_num(y.float(), nan=-9.0))
    out = torch.full((9, 6, 64), 5.0, dtype=torch.bfloat16, device="cuda:0")
    b.cb.ss_cache_read(b.desc, 9, b.cu["new"], b.start, b.dev_table, *b.store, out[:, 2:4], out[:, 4:], 384, 64, b.stream())
    want = a.read(9, a.cu["new"], a.start)
    assert torch.equal(out[:, 2:4], want[0]) and torch.equal(out[:, 4:], want[1]) and bool((out[:, :2] == 5.0).all())


# past, new, H, HK, D, page
ATTN = {
    "first_token": ([0], [1], 1, 1, 64, 16),
    "one_of_each": ([0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 255, 256, 257], [1] * 14, 8, 2, 128, 16),
    "equal_heads": ([100, 300], [1, 1], 4, 4, 128, 64),
    "wide_group": ([70, 500], [1, 1], 40, 1, 128, 32),
    "few_tokens": ([50, 0, 200], [3, 7, 1], 12, 4, 128, 16),
    "few64": ([50, 0, 200, 33], [3, 7, 0, 8], 16, 2, 64, 8),
    "group_of_three": ([129, 64], [5, 2], 6, 2, 64, 128),
    "many_rows": ([40, 333], [64, 31], 8, 1, 128, 16),
    "long_rows": ([700], [64], 16, 2, 128, 64),
    "big_page": ([1500, 3], [2, 2], 4, 2, 128, 1024),
    "long": ([2900, 10, 777], [1, 1, 1], 8, 2, 128, 16),
    "empty_sequences": ([0, 40, 0], [0, 2, 0], 4, 2, 128, 16),
    "many_sequences": ([(37 * i) % 90 for i in range(150)], [i % 3 for i in range(150)], 4, 1, 64, 8),
    "pieces": ([600, 5, 0, 1300, 90, 513], [3, 1, 2, 4, 0, 1], 8, 2, 128, 16),
    "pieces_of_many": ([(61 * i) % 700 for i in range(100)], [i % 4 for i in range(100)], 4, 2, 64, 16),
    "groups_of_rows": ([600, 5, 900, 1300, 0], [40, 3, 0, 64, 33], 8, 2, 128, 16),
    "groups64": ([33, 1100, 640], [10, 64, 17], 24, 3, 64, 32),
    "up_to_64_rows": ([800, 20, 450], [15, 16, 9], 12, 3, 128, 8),
    "more_heads_than_work_groups": ([130, 3], [1, 1], 514, 514, 64, 1024),
}


@pytest.mark.parametrize("tree", [False, True], ids=["row", "tree"])
@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("name", ATTN)
def test_attention_against_the_oracle(name, fmt, tree):
    import torch
    from cache_cases import Cache
    past, new, H, HK, D, page = ATTN[name]
    print(f"cache attention {name} {fmt} tree={tree}", flush=True)
    c = Cache(len(name), past, new, H, HK, D, fmt, page)
    if tree:
        c.plant_tree(5, empty_rows=True)
    c.write("past")
    c.write("new")
    c.attn()
    torch.cuda.synchronize()
    c.check_attention(c.want_values())


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("gain,scale", [(8.0, None), (1.0, 0.0), (1.0, -0.3)])
def test_attention_of_peaked_and_flat_rows(fmt, gain, scale):
    import torch
    from cache_cases import Cache
    print(f"cache attention data {fmt} {gain} {scale}", flush=True)
    c = Cache(41, [600, 90], [4, 1], 8, 2, 128, fmt, 32, gain=gain, scale=scale, pad=8)
    c.write("past")
    c.write("new")
    c.attn()
    torch.cuda.synchronize()
    c.check_attention(c.want_values())


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
def test_pages_that_are_not_there(fmt):
    """Table entries outside the pool, and lengths beyond the table: not written, read as zeros, not seen; nothing else changes."""
    import torch
    from cache_cases import Cache
    print(f"cache bad pages {fmt}", flush=True)
    c = Cache(43, [200, 100, 40], [6, 6, 6], 4, 2, 128, fmt, 16)
    for at, bad in (((0, 3), -1), ((0, 7), c.n_pages), ((1, 6), -2 ** 31), ((2, 0), 2 ** 31 - 1), ((2, 1), -7), ((2, 2), 1 << 20)):
        c.table[at] = bad
    c.dev_table.copy_(torch.from_numpy(c.table))
    c.write("past")
    c.write("new")
    c.attn()
    cu_all = torch.from_numpy(np.concatenate([[0], np.cumsum(c.lens)]).astype(np.int32)).cuda()
    K = c.read(int(cu_all[-1]), cu_all, None)[0]
    torch.cuda.synchronize()
    values = c.want_values()
    c.check_attention(values)
    from oracle import cache as oc
    for b in range(3):
        for pos in range(int(c.lens[b])):
            at = oc.find(c.table, c.n_pages, 16, b, pos)
            row = K[int(cu_all[b]) + pos].float().cpu().numpy()
            want = values[0][at[0], :, at[1]] if at else np.zeros((2, 128))
            np.testing.assert_allclose(row, want, rtol=2 ** -8, atol=0)


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
def test_lengths_beyond_the_table(fmt):
    """The positions behind the table's last page are not there, the new tokens among them."""
    import torch
    from cache_cases import Cache
    print(f"cache long lengths {fmt}", flush=True)
    c = Cache(44, [26, 42], [6, 6], 4, 2, 128, fmt, 16)  # pages that are full
    c.write("past")
    c.write("new")
    c.lens[:] = [35, 54]
    seen = {}
    for lens in ([35, 54], [54, 54], [2 ** 31 - 1, 2 ** 31 - 1], [-4, -2 ** 31], [2, 0]):
        c.dev_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.Y.fill_(float("nan"))
        c.attn()
        torch.cuda.synchronize()
        seen[lens[0]] = c.Y.clone(), c.lse.clone()
        if lens[0] == 35:
            c.check_attention(c.want_values())
    assert torch.equal(seen[54][0][:6], seen[2 ** 31 - 1][0][:6]) and torch.equal(seen[54][1], seen[2 ** 31 - 1][1])
    assert bool((seen[-4][0] == 0).all()) and bool((seen[-4][1] == float("-inf")).all())
    assert not torch.isnan(seen[2][0]).any()


def test_more_new_tokens_than_said():
    """Rows from max_new on are left as they were."""
    import torch
    from cache_cases import Cache
    print("cache max_new", flush=True)
    c = Cache(45, [30, 60], [9, 4], 4, 2, 64, "fp8", 16, max_new=5)
    c.write("past")
    c.write("new")
    c.attn()
    torch.cuda.synchronize()
    c.check_attention(c.want_values())


def test_a_pool_beyond_32_bits():
    """More than 2^32 bytes of codes and rows at both ends of the pool."""
    import torch
    from cache_cases import Cache
    from paper_2301_08984_amd import cache_binding as cb
    print("cache large pool", flush=True)
    small = Cache(47, [70, 33], [2, 1], 8, 4, 128, "int8", 128)
    big_pages = (1 << 32) // (128 * 4 * 128) + 9
    for c in (small,):
        c.write("past")
        c.write("new")
        c.attn()
    big = Cache(47, [70, 33], [2, 1], 8, 4, 128, "int8", 128)
    big.n_pages = big_pages
    big.table[:, 0] = [big_pages - 1, 0]
    big.dev_table.copy_(torch.from_numpy(big.table))
    big.desc = cb.make_desc(big_pages, 128, 4, 128, 2, 2, big.max_pages)
    codes, scales = cb.ss_cache_bytes(big.desc)
    assert codes > 1 << 32
    big.store = [torch.empty(codes, dtype=torch.uint8, device="cuda:0"), torch.empty(scales // 4, device="cuda:0"),
                 torch.empty(codes, dtype=torch.uint8, device="cuda:0"), torch.empty(scales // 4, device="cuda:0")]
    big.write("past")
    big.write("new")
    big.attn()
    torch.cuda.synchronize()
    assert torch.equal(big.Y, small.Y) and torch.equal(big.lse, small.lse)


def test_captured_decoding():
    """A graph of one decoding step (write, attention), replayed while lengths, pages and tokens change."""
    import torch
    from cache_cases import Cache
    from oracle import cache as oc
    print("cache captured", flush=True)
    steps = 5
    c = Cache(49, [95, 30, 700], [1, 1, 1], 8, 2, 128, "fp8", 16, room=4)
    for b, n in enumerate((96, 31, 701)):  # pages for the steps to come
        have = -(-n // 16)
        free = [p for p in range(c.n_pages) if p not in c.table]
        c.table[b, have:have + 1] = free[:1]
    c.dev_table.copy_(torch.from_numpy(c.table))
    c.write("past")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        c.write("new")
        c.attn()
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    values = None
    for step in range(steps):
        for x in (*c.kv["new"], c.Q):
            x.copy_(torch.randn(x.shape, generator=gen, device="cuda:0"))
        c.Y.fill_(float("nan"))
        c.ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        got, got_lse = c.Y.clone(), c.lse.clone()
        c.write("new")
        c.attn()
        torch.cuda.synchronize()
        assert torch.equal(got, c.Y) and torch.equal(got_lse, c.lse), step
        if values is None:
            values = c.want_values()
        for b in range(3):  # what earlier steps wrote stays in the oracle's cache
            pos = int(c.start[b])
            for old, x in zip(values, c.host_kv("new")):
                old[c.table[b, pos // 16], :, pos % 16] = oc.values(x[b], c.fmt)
        c.check_attention(values)
        c.start += 1
        c.dev_lens += 1
        c.lens += 1


def test_prompt_then_turn_then_tree():
    """The operators as a server uses them: a prompt's attention and its rows into the cache, a second turn over what is read back, a tree
    of drafts over the cache; each against the oracle."""
    import torch
    from cache_cases import Cache
    from packed_cases import Packed
    from oracle import packed as op
    from packed_cases import off
    from paper_2301_08984_amd import packed_binding as pb
    print("cache run together", flush=True)
    H, HK, D = 8, 2, 128
    c = Cache(51, [90, 40], [20, 33], H, HK, D, "fp8", 16)
    prompt = Packed(52, [90, 40], H, HK, D)
    prompt.K.copy_(c.kv["past"][0])
    prompt.V.copy_(c.kv["past"][1])
    prompt.fwd()
    c.write("past")
    c.write("new")
    lens = [110, 73]
    cu_all = torch.tensor([0, 110, 183], dtype=torch.int32, device="cuda:0")
    K, V = c.read(183, cu_all, None)
    Y = torch.full((53, H, D), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    lse = torch.full((H, 53), float("nan"), device="cuda:0")
    d = pb.make_desc(53, 2, H, HK, D, 0, HK, 1, Tk=183)
    pb.ss_packed_fwd(d, c.Q, K, V, c.cu["new"], cu_all, Y, lse, None, 0, c.stream())
    c.attn()
    row = c.Y.clone()
    c.plant_tree(6)
    c.attn()
    torch.cuda.synchronize()
    prompt.check(prompt.oracle(), ("Y", "lse"))
    values = c.want_values()
    c.check_attention(values)
    ref = op.attention(c.Q.float().cpu().numpy(), K.float().cpu().numpy(), V.float().cpu().numpy(), np.array([0, 20, 53]), np.array([0] + list(np.cumsum(lens))),
                       c.scale)
    for got in (Y, row):  # a row of new tokens over the cache is the second turn
        got = got.float().cpu().numpy().astype(np.float64)
        assert off(got, ref["Y"]) <= 2 * op.U and np.all(np.abs(got - ref["Y"]) <= op.bounds(ref, "Y") + 2.0 ** -13 * ref["Y_mag"])
