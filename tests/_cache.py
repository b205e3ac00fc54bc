"""Shared helpers of the bounded-cache GPU tests (imported by test modules only):
caches in any stride order or paged, the calls, and derived error bounds."""
from __future__ import annotations

import numpy as np
import torch

from oracle import cache_oracle as CO
from paper_2605_31457_amd import vp

DEV = "cuda:0"
EPS = 2.0 ** -24  # half a step of float32, relative


def torch_dtype(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def rounded(x, dtype):
    """x as the stored type holds it, in float64."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch_dtype(dtype)).double().numpy()


class Caches:
    """K and V of a batch on the device. K, V: float64 [B][Hkv, cap, d] as stored.
    order: "bhs" (heads before rows), "bsh" (rows before heads) or "pad" (rows 16
    elements further apart); page > 0: blocks of `page` rows in a random order, two
    spare blocks. `fill` lies wherever no row does."""

    def __init__(self, K, V, dtype, order="bhs", page=0, seed=0, fill=0.0):
        B, Hkv, cap, d = K.shape
        self.dtype, self.page, self.cap = dtype, page, cap
        td = torch_dtype(dtype)
        if page:
            n = -(-cap // page)
            self.table = torch.from_numpy(np.random.default_rng(seed).permutation(B * n + 2)[:B * n].reshape(B, n))
            shape = (B * n + 2, Hkv, page, d)
        else:
            self.table, shape = None, (B, Hkv, cap, d)
        self.K, self.V = (self._empty(shape, order, td, fill) for _ in range(2))
        self.table = None if self.table is None else self.table.to(torch.int32).to(DEV)
        self.put(K, V)

    @staticmethod
    def _empty(shape, order, td, fill):
        n, h, s, d = shape
        if order == "bsh":
            return torch.full((n, s, h, d), fill, dtype=td, device=DEV).transpose(1, 2)
        if order == "pad":
            return torch.full((n, h, s, d + 16), fill, dtype=td, device=DEV)[..., :d]
        return torch.full(shape, fill, dtype=td, device=DEV)

    def put(self, K, V):
        for dst, src in ((self.K, K), (self.V, V)):
            src = torch.from_numpy(np.ascontiguousarray(src)).to(torch_dtype(self.dtype)).to(DEV)
            if not self.page:
                dst.copy_(src)
                continue
            for b in range(src.shape[0]):
                for j in range(self.table.shape[1]):
                    rows = src[b, :, j * self.page:(j + 1) * self.page]
                    dst[int(self.table[b, j]), :, :rows.shape[1]] = rows

    def get(self):
        """(K, V) as float64 [B, Hkv, cap, d]."""
        out = []
        for x in (self.K, self.V):
            if self.page:
                t = self.table.long()
                x = x[t].permute(0, 2, 1, 3, 4).reshape(t.shape[0], x.shape[1], -1, x.shape[3])[:, :, :self.cap]
            out.append(x.double().cpu().numpy())
        return out

    def shape(self, Hq, T=1, scope=0, cap=None):
        Hkv, d = self.K.shape[1], self.K.shape[3]
        B = self.table.shape[0] if self.page else self.K.shape[0]
        sb, sh, ss, _ = self.K.stride()
        return vp.vp_shape(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d,
                           dtype=vp.VP_BF16 if self.dtype == "bf16" else vp.VP_F32, max_seq_len=cap or self.cap,
                           max_vis=1, max_segs=256, k_cap=1, block_size=self.page, scope=scope, n_queries=T,
                           kv_stride_b=sb, kv_stride_h=sh, kv_stride_s=ss)

    def layout(self, seq_len, off=None, seg=None):
        p = lambda t: None if t is None else t.data_ptr()
        return vp.vp_layout(seq_len=p(seq_len), vis_seg_off=p(off), vis_seg=p(seg), block_table=p(self.table))


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def attention(c: Caches, q, lens, window, n_sink, sums=None, scale=0.0, stream=None):
    """One vp_window_decode_attn call; q: device [B, T, Hq, d]. Returns out as a tensor."""
    B, T, Hq, d = q.shape
    shape, w = c.shape(Hq, T), vp.vp_window(window=window, n_sink=n_sink, sm_scale=scale)
    seq_len = i32(lens)
    out = torch.full_like(q, 7.0)
    nbytes = vp.vp_window_workspace_size(shape, w, sums is not None)
    ws = torch.full((nbytes + 64,), 0xff, dtype=torch.uint8, device=DEV)
    vp.vp_window_decode_attn(shape, c.layout(seq_len), w, q, c.K, c.V, sums, out, ws, nbytes, stream)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0xff).all())  # nothing past the size that was asked for
    return out


def weight_error(r: CO.WindowResult, d, n, TG):
    """Relative error of an attention weight: z is a sum of d products in float32
    (any order: at most d roundings of partial sums no larger than span) and is
    scaled by a rounded constant; 2^x is a step off or two, from an argument
    rounded at |z| and at |z - m| <= 2 span; the normaliser adds n / 32 tile sums
    per wave in order, 32 terms each, and the joins of waves and parts."""
    span = float(r.span.max()) if r.span.size else 0.0
    z = (d + 2) * EPS * span + 4 * EPS * 1.45 * 2 * span
    return 2 * z + (n / 32 + 32 + 16) * EPS + 8 * EPS


def assert_attention(got, r: CO.WindowResult, dtype, n, ctx=""):
    """out [T, Hq, d] against the reference: the weights' error, the value sums'
    float32 order, the split weights (bf16: 16 bits) and half a step of the type."""
    T, Hq, d = r.out.shape
    e = weight_error(r, d, n, T * Hq) + (n / 32 + 32 + 16) * EPS + (2.0 ** -15 if dtype == "bf16" else 0.0)
    step = 2.0 ** -8 if dtype == "bf16" else EPS
    bound = e * r.spread + step * (np.abs(r.out) + e * r.spread) + 1e-37
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got)), ctx
    worst = np.max(np.abs(got - r.out) / bound)
    assert worst <= 1.0, f"{ctx}: {worst:.2f} times the bound"


def assert_sums(got, before, r: CO.WindowResult, L, T, n, d, TG, ctx=""):
    """attn_sum [Hkv, cap] after the call: rows seen by a query have their weights
    added (new rows from zero), everything else keeps its bits."""
    Hkv, cap = before.shape
    seen = np.zeros(cap, bool)
    seen[:L] = r.seen.any(0)
    assert np.array_equal(got[:, ~seen], before[:, ~seen], equal_nan=True), f"{ctx}: rows that no query sees"
    want = before.astype(np.float64).copy()
    want[:, max(0, L - T):L] = 0.0
    add = np.zeros((Hkv, cap))
    add[:, :L] = r.weight
    want += add
    # the weights' error, their sum over T*G query rows, and the addition's rounding
    bound = (weight_error(r, d, n, TG) + (TG + 1) * EPS) * add + EPS * np.abs(want) + 1e-37
    err = np.abs(got - want)[:, seen]
    assert np.all(err <= bound[:, seen]), f"{ctx}: sums {np.max(err / bound[:, seen]):.2f} times the bound"
