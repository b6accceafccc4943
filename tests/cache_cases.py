"""Shared helpers of the tests of the paged cache: device arrays with garbage wherever no row lies, the calls, the oracle."""
import math

import numpy as np

from oracle import cache as oc
from oracle import packed as op
from packed_cases import off, starts

FORMATS = {"bf16": 0, "fp8": 1, "int8": 2}


class Cache:
    """A cache that `past` tokens of every sequence were written into, then the `new` ones, by ss_cache_write; pages in no order,
    garbage (NaN, the largest codes) in every other slot."""

    def __init__(self, seed, past, new, H, HK, D, fmt, page, *, scale=None, spare=3, room=0, gain=1.0, max_new=None, pad=0):
        import torch
        from paper_2301_08984_amd import cache_binding as cb
        self.cb, self.torch, self.fmt, self.page, self.D, self.H, self.HK = cb, torch, FORMATS[fmt], page, D, H, HK
        rng = np.random.default_rng(seed)
        self.past, self.new, n_seq = list(past), list(new), len(past)
        pages = [-(-(p + n) // page) for p, n in zip(past, new)]
        self.n_pages, self.max_pages = sum(pages) + spare, max(max(pages), 1) + room
        order = rng.permutation(self.n_pages)
        self.table = np.full((n_seq, self.max_pages), self.n_pages + 9, np.int32)  # entries that are not used: no page
        for b, p in enumerate(pages):
            self.table[b, :p], order = order[:p], order[p:]
        self.scale = float(np.float32(1 / math.sqrt(D) if scale is None else scale))
        self.dev_table = torch.from_numpy(self.table).cuda()
        self.desc = cb.make_desc(self.n_pages, page, HK, D, self.fmt, n_seq, self.max_pages)
        codes, scales = cb.ss_cache_bytes(self.desc)
        self.store = []
        for _ in range(2):
            c = torch.full((codes,), 0xFF if fmt == "bf16" else 0x7F, dtype=torch.uint8, device="cuda:0")  # NaN (int8: 127)
            s = torch.full((scales // 4,), float("nan"), device="cuda:0") if scales else None
            self.store += [c, s]
        bf16 = lambda *shape: torch.from_numpy(rng.normal(size=shape).astype(np.float32)).cuda().bfloat16()  # noqa: E731
        self.kv = {w: (bf16(sum(lens), HK, D), bf16(sum(lens), HK, D)) for w, lens in (("past", past), ("new", new))}
        self.cu = {w: torch.from_numpy(starts(lens)).cuda() for w, lens in (("past", past), ("new", new))}
        self.start = torch.from_numpy(np.array(past, np.int32)).cuda()
        self.lens = np.array([p + n for p, n in zip(past, new)], np.int32)
        self.dev_lens = torch.from_numpy(self.lens).cuda()
        T = sum(new)
        self.max_new = min(max(max(new), 1), 64) if max_new is None else max_new
        full = torch.full((T, H, D + pad), float("nan"), dtype=torch.bfloat16, device="cuda:0")
        full[..., :D] = bf16(T, H, D) * gain
        self.Q = full[..., :D]
        self.Y = torch.full((T, H, D + pad), float("nan"), dtype=torch.bfloat16, device="cuda:0")[..., :D]
        self.lse = torch.full((H, T), float("nan"), device="cuda:0")
        self.tree = None
        if T:
            self.attn_desc = cb.make_attn_desc(T, H, self.max_new, D, scale=self.scale, q_stride_t=H * (D + pad), q_stride_h=D + pad,
                                               y_stride_t=H * (D + pad), y_stride_h=D + pad)
            self.ws = torch.full((max(cb.ss_cache_attn_workspace_bytes(self.desc, self.attn_desc), 256),), 0xFF, dtype=torch.uint8, device="cuda:0")

    def stream(self):
        return self.torch.cuda.current_stream().cuda_stream

    def write(self, which):
        K, V = self.kv[which]
        if K.shape[0]:
            self.cb.ss_cache_write(self.desc, K.shape[0], K, V, self.HK * self.D, self.D, self.cu[which], None if which == "past" else self.start,
                                   self.dev_table, *self.store, self.stream())

    def read(self, T, cu, start):
        """-> K, V [T, HK, D] with NaN where nothing was written."""
        K, V = (self.torch.full((T, self.HK, self.D), float("nan"), dtype=self.torch.bfloat16, device="cuda:0") for _ in range(2))
        self.cb.ss_cache_read(self.desc, T, cu, start, self.dev_table, *self.store, K, V, self.HK * self.D, self.D, self.stream())
        return K, V

    def attn(self):
        self.cb.ss_cache_attn(self.desc, self.attn_desc, self.Q, self.cu["new"], self.dev_lens, self.tree, self.dev_table, *self.store, self.Y,
                              self.lse, self.ws, self.ws.numel(), self.stream())

    def plant_tree(self, seed, empty_rows=False):
        """Random sets of visible drafts (a tree's are among them); with `empty_rows` some that see none."""
        rng = np.random.default_rng(seed)
        bits = []
        for n in self.new:
            rows = []
            for i in range(n):
                parent = int(rng.integers(-1, i)) if i else -1
                rows.append((rows[parent] if parent >= 0 else 0) | 1 << i)
            if empty_rows and n:
                rows[int(rng.integers(0, n))] = 0
            bits += rows
        self.bits = bits
        signed = np.array([b - (1 << 64) if b >> 63 else b for b in bits], np.int64)
        self.tree = self.torch.from_numpy(signed).cuda()

    def host_kv(self, which):
        return [x.float().cpu().numpy() for x in self.kv[which]]

    def want_values(self):
        """[n_pages, HK, page, D] of K and of V as the written rows say, zeros elsewhere, from the tokens alone."""
        out = [np.zeros((self.n_pages, self.HK, self.page, self.D)) for _ in range(2)]
        for which, lens, first in (("past", self.past, [0] * len(self.past)), ("new", self.new, self.past)):
            at = 0
            both = [oc.values(x, self.fmt) for x in self.host_kv(which)]
            for b, n in enumerate(lens):
                for i in range(n):
                    place = oc.find(self.table, self.n_pages, self.page, b, first[b] + i)
                    if place:
                        for o, x in zip(out, both):
                            o[place[0], :, place[1]] = x[at + i]
                at += n
        return out

    def check_attention(self, values):
        cu = self.cu["new"].cpu().numpy()
        ref = oc.attention(self.Q.float().cpu().numpy(), *values, self.table, self.page, cu, self.lens, self.bits if self.tree is not None else None,
                           self.scale, self.max_new)
        got, want = self.Y.float().cpu().numpy().astype(np.float64), ref["Y"]
        keep = ~np.isnan(want)
        assert np.isnan(got[~keep]).all() and not np.isnan(got[keep]).any(), "rows written or left out"
        # (8 bits: the codes' products are summed with an offset of up to 128 a code, in fp32: 2^-17 of their size)
        bar = op.bounds(ref, "Y") + (2.0 ** -13 if self.fmt else 0.0) * ref["Y_mag"] + 1e-30
        assert float(np.max((np.abs(got - want) / bar)[keep], initial=0.0)) <= 1.0
        assert off(got[keep], want[keep]) <= 2 * op.U
        l, w = self.lse.cpu().numpy().astype(np.float64), ref["lse"]
        there = ~np.isnan(w)
        assert np.isnan(l[~there]).all()
        inf = there & np.isinf(w)
        assert np.array_equal(l[inf], w[inf])
        fine = there & ~inf
        assert np.all(np.abs(l - w)[fine] <= (2.0 ** -17 if self.fmt == 2 else 2.0 ** -20) * (1 + np.abs(w) + ref["near"])[fine])
