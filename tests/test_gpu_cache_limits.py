"""Attention over the cache at the end of the longest table: positions up to 2^31 - 64, all but the last pages of which are not there."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [2 ** 31 - 64, 2 ** 31 - 65, 2 ** 31 - 129])
@pytest.mark.parametrize("H,new", [(1, 1), (2, 17), (2, 40)], ids=["a_row", "34_rows", "80_rows"])
def test_the_last_positions_of_the_longest_table(H, new, lens):
    """The keys of the last five pages alone decide, as they do in a table of five pages.  (What the two calls round to bf16 are P, at maxima that may differ,
    and the result: half a step each.)"""
    import torch
    from paper_2301_08984_amd import cache_binding as cb
    print(f"cache last positions {H} {new} {lens}", flush=True)
    page, pages, D = 64, 5, 64
    entries = 2 ** 31 // page - 1
    rng = np.random.default_rng(5)
    small = cb.make_desc(pages, page, 1, D, cb.SS_CACHE_INT8, 1, pages)
    big = cb.make_desc(pages, page, 1, D, cb.SS_CACHE_INT8, 1, entries)
    codes, scales = cb.ss_cache_bytes(small)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    store = []
    for _ in range(2):
        store += [torch.randint(-127, 128, (codes,), generator=gen, device="cuda:0").to(torch.int8), torch.full((scales // 4,), 0.02, device="cuda:0")]
    order = torch.from_numpy(rng.permutation(pages).astype(np.int32)).cuda()
    table = torch.full((1, entries), -1, dtype=torch.int32, device="cuda:0")
    table[0, -pages:] = order
    Q = torch.randn((new, H, D), generator=gen, device="cuda:0").bfloat16()
    cu = torch.tensor([0, new], dtype=torch.int32, device="cuda:0")
    st = torch.cuda.current_stream().cuda_stream
    got = []
    for desc, tab, n in ((small, order.reshape(1, -1).contiguous(), lens - (entries - pages) * page), (big, table, lens)):
        attn = cb.make_attn_desc(new, H, new, D)
        need = cb.ss_cache_attn_workspace_bytes(desc, attn)
        ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda:0")
        Y, lse = torch.full_like(Q, float("nan")), torch.full((H, new), float("nan"), device="cuda:0")
        dev_lens = torch.tensor([n], dtype=torch.int32, device="cuda:0")
        cb.ss_cache_attn(desc, attn, Q, cu, dev_lens, None, tab, *store, Y, lse, ws, ws.numel(), st)
        torch.cuda.synchronize()
        got.append((Y.double(), lse.double()))
    (y, l), (Y, L) = got
    assert not torch.isnan(Y).any() and not torch.isnan(L).any()
    assert float((L - l).abs().max()) <= 2.0 ** -17 * (1 + float(l.abs().max()))
    # |v| <= 127 * 0.02 = 2.54, of which a probability takes its share: at most that
    assert float((Y - y).abs().max()) <= 2 * 2.0 ** -8 * (2.54 + float(y.abs().max()))
    assert float((Y - y).norm() / y.norm()) <= 4 * 2.0 ** -8
