"""Shared helpers of the tests of packed attention and of the cache: device tensors, the calls, and the comparison.

Inputs are bf16 numbers.  Two bars for every floating output, both derived from what is rounded:
  * element by element: half a step of bf16 (2^-8 of a value) for the rounded operand of the last product, against the sum
    of the products' magnitudes, and for the result (oracle.packed.bounds);
  * the 2-norm of the difference over that of the result: these roundings are at most half a step each and have no common
    sign, so 2 half-steps for Y (P, Y) and 3 for a gradient (P or dS, Delta, the result) are above what they can add up to.  It
    notices a key left out, which the first bar may not."""
import math

import numpy as np

from oracle import packed as op


def off(x, ref):
    norm = np.linalg.norm(ref)
    return float(np.linalg.norm(x - ref) / norm) if norm else float(np.linalg.norm(x))


def starts(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32)


class Packed:
    """One operator: Q, K, V, dY as slices of buffers filled with NaN, outputs too, `before` and `behind` rows of no sequence."""

    def __init__(self, seed, lens_q, H, HK, D, lens_k=None, *, scale=None, before=0, behind=0, pad=0, peaked=1.0, offset=0.0, share=None, k=1):
        import torch
        from paper_2301_08984_amd import packed_binding as pb
        self.pb, self.torch = pb, torch
        rng = np.random.default_rng(seed)
        self.cu_q = starts(lens_q, before)
        self.cu_k = self.cu_q if lens_k is None else starts(lens_k, before)
        Tq, Tk = int(self.cu_q[-1]) + behind, int(self.cu_k[-1]) + behind
        self.H, self.HK, self.D, self.k = H, HK, D, k
        self.lo, self.hi = (0, HK) if share is None else share
        self.scale = float(np.float32(1 / math.sqrt(D) if scale is None else scale))

        def make(T, heads, cu, gain=1.0, shift=0.0):
            full = torch.full((T, heads, D + pad), float("nan"), dtype=torch.bfloat16, device="cuda:0")
            x = torch.from_numpy((rng.normal(size=(int(cu[-1] - cu[0]), heads, D)) * gain + shift).astype(np.float32)).cuda().bfloat16()
            full[int(cu[0]):int(cu[-1]), :, :D] = x
            return full[..., :D]
        self.Q, self.dY = make(Tq, H, self.cu_q, peaked), make(Tq, H, self.cu_q, 1.0, offset)
        self.K, self.V = make(Tk, HK, self.cu_k), make(Tk, HK, self.cu_k, 1.0, offset)
        empty = lambda like: torch.full_like(like, float("nan"), memory_format=torch.contiguous_format)  # noqa: E731
        # (outputs with the strides of their inputs)
        same = lambda x, heads, T: torch.full((T, heads, D + pad), float("nan"), dtype=torch.bfloat16, device="cuda:0")[..., :D]  # noqa: E731
        self.Y, self.dQ, self.dK, self.dV = same(0, H, Tq), same(0, H, Tq), same(0, HK, Tk), same(0, HK, Tk)
        self.lse = torch.full((H, Tq), float("nan"), device="cuda:0")
        self.dev_q = torch.from_numpy(self.cu_q).cuda()
        self.dev_k = None if lens_k is None else torch.from_numpy(self.cu_k).cuda()
        st = dict(q_stride_t=self.Q.stride(0), q_stride_h=self.Q.stride(1), k_stride_t=self.K.stride(0), k_stride_h=self.K.stride(1),
                  y_stride_t=self.Y.stride(0), y_stride_h=self.Y.stride(1))
        self.desc = pb.make_desc(Tq, len(lens_q), H, HK, D, self.lo, self.hi, k, Tk=Tk, scale=self.scale, **st)
        need = pb.ss_packed_workspace_bytes(self.desc)[1]
        self.ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda:0")

    def stream(self):
        return self.torch.cuda.current_stream().cuda_stream

    def fwd(self):
        self.pb.ss_packed_fwd(self.desc, self.Q, self.K, self.V, self.dev_q, self.dev_k, self.Y, self.lse, None, 0, self.stream())

    def bwd(self, keep):
        self.pb.ss_packed_bwd(self.desc, self.Q, self.K, self.V, self.dev_q, self.dev_k, self.Y if keep else None, self.dY,
                              self.lse if keep else None, self.dQ, self.dK, self.dV, self.ws, self.ws.numel(), self.stream())

    def host(self, name):
        return getattr(self, name).float().cpu().numpy().astype(np.float64)

    def oracle(self):
        Q, K, V, dY = (self.host(n) for n in ("Q", "K", "V", "dY"))
        return op.attention(Q, K, V, self.cu_q, self.cu_k, self.scale, dY)

    def check(self, ref, names=("Y", "lse", "dQ", "dK", "dV")):
        """Against the oracle inside the share's sequences; outside nothing may have been written."""
        G = self.H // self.HK
        for name in names:
            got, want = self.host(name), ref[name].copy()
            heads = slice(self.lo, self.hi) if name in ("dK", "dV") else slice(self.lo * G, self.hi * G)
            axis = (heads,) if name == "lse" else (slice(None), heads)
            keep = np.zeros(want.shape, bool)
            keep[axis] = True
            keep &= ~np.isnan(want)
            assert np.isnan(got[~keep]).all(), (name, "written outside the share or the sequences")
            if name == "lse":
                same = np.isinf(want) & keep
                assert np.array_equal(got[same], want[same]), name
                keep &= ~np.isinf(want)
                # fp32: the score's products (24 bits each, against their magnitudes), the exponentials, their sum
                err, bar = np.abs(got - want)[keep], (2.0 ** -20 * (1 + np.abs(want) + ref["near"]))[keep]
            else:
                err, bar = np.abs(got - want)[keep], op.bounds(ref, name)[keep] + 1e-30
                if keep.any():
                    assert off(got[keep], want[keep]) <= (2 if name == "Y" else 3) * op.U, (name, off(got[keep], want[keep]))
            assert not np.isnan(got[keep]).any(), (name, "not written")
            worst = float(np.max(err / bar, initial=0.0))
            assert worst <= 1.0, (name, worst)
