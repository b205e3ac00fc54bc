"""Shared helpers of the tests of appending and of 4-bit caches (imported by test modules only)."""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from oracle import kv4_oracle as KO
from paper_2605_31457_amd import vp
from _cache import DEV, EPS, Caches, i32, rounded, torch_dtype


def cos_sin(n_pos, rot, seed=0):
    """float32 [n_pos, rot]: cosines, then sines, of usual angles."""
    a = np.arange(n_pos)[:, None] * (1e4 ** (-np.arange(0, rot, 2) / rot))
    return np.concatenate([np.cos(a + seed), np.sin(a + seed)], 1).astype(np.float32)


class Four:
    """A 4-bit cache on the device, contiguous or paged; `fill` lies wherever no row does.
    The K and V strides leave room between heads where `gap` says so."""

    def __init__(self, B, Hkv, cap, d, page=0, seed=0, fill=0xEE, gap=0, table=None):
        self.page, self.cap, self.d = page, cap, d
        n, rows = (B, -(-cap // 16) * 16 + gap) if not page else (B * -(-cap // page) + 2, page + gap)
        self.table = table
        if page and table is None:
            blocks = -(-cap // page)
            self.table = torch.from_numpy(np.random.default_rng(seed).permutation(n)[:B * blocks].reshape(B, blocks)).to(torch.int32).to(DEV)
        self.codes = [torch.full((n, Hkv, rows, d // 2), fill, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.scales = [torch.full((n, Hkv, rows, d // 32), fill, dtype=torch.uint8, device=DEV) for _ in range(2)]

    def struct(self):
        (kc, vc), (ks, vs) = self.codes, self.scales
        return vp.vp_kv4(k_codes=kc.data_ptr(), k_scales=ks.data_ptr(), v_codes=vc.data_ptr(), v_scales=vs.data_ptr(),
                         code_stride_b=kc.stride(0), code_stride_h=kc.stride(1), scale_stride_b=ks.stride(0),
                         scale_stride_h=ks.stride(1))

    def _rows(self, x, L):
        """[B, Hkv, L, ...] of a plane array."""
        if self.page:
            t = self.table.long()
            x = x[t][:, :, :, :self.page].permute(0, 2, 1, 3, 4).reshape(t.shape[0], x.shape[1], -1, x.shape[3])
        return x[:, :, :L]

    def put(self, K, V):
        """Rows [B][Hkv, L, d] in float64, quantised by the reference."""
        for x, codes, scales in zip((K, V), self.codes, self.scales):
            for b in range(len(x)):
                c, s = KO.quantise(x[b])
                c = torch.from_numpy(c[..., 0::2] | (c[..., 1::2] << 4)).to(DEV)
                s = torch.from_numpy(s).to(DEV)
                for src, dst in ((c, codes), (s, scales)):
                    if not self.page:
                        dst[b, :, :src.shape[1]] = src
                        continue
                    for j in range(-(-src.shape[1] // self.page)):
                        part = src[:, j * self.page:(j + 1) * self.page]
                        dst[int(self.table[b, j]), :, :part.shape[1]] = part

    def get(self, L):
        """(K, V) as float64 [B, Hkv, L, d], by the reference's reading of the bytes."""
        out = []
        for codes, scales in zip(self.codes, self.scales):
            c = self._rows(codes, L).cpu().numpy()
            s = self._rows(scales, L).cpu().numpy()
            c = np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], -1)
            out.append(KO.decode(c, s))
        return out

    def shape(self, Hq, dtype, T=1, cap=None):
        n, Hkv = self.codes[0].shape[:2]
        B = self.table.shape[0] if self.page else n
        cap = cap or self.cap
        return vp.vp_shape(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=self.d,
                           dtype=vp.VP_BF16 if dtype == "bf16" else vp.VP_F32, max_seq_len=cap, max_vis=1, max_segs=1,
                           k_cap=1, block_size=self.page, scope=0, n_queries=T, kv_stride_b=0, kv_stride_h=0,
                           kv_stride_s=self.d)

    def layout(self, seq_len):
        return vp.vp_layout(seq_len=seq_len.data_ptr(), vis_seg_off=None, vis_seg=None,
                            block_table=None if self.table is None else self.table.data_ptr())


class New:
    """New tokens on the device: q [n, Hq, d], k, v [n, Hkv, d] (float64, as stored), as
    columns of one array or apart."""

    def __init__(self, rng, n, Hq, Hkv, d, dtype, fused=True, queries=True, scale=1.0):
        x = rounded(rng.standard_normal((n, Hq + 2 * Hkv, d)) * scale, dtype)
        self.set(x, Hq, Hkv, dtype, fused, queries)

    def set(self, x, Hq, Hkv, dtype, fused=True, queries=True):
        self.n, self.dtype, self.queries = x.shape[0], dtype, queries
        self.q, self.k, self.v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        self.dev = torch.from_numpy(x).to(torch_dtype(dtype)).to(DEV)
        parts = self.dev[:, :Hq], self.dev[:, Hq:Hq + Hkv], self.dev[:, Hq + Hkv:]
        self.parts = parts if fused else tuple(p.contiguous() for p in parts)

    def struct(self, new_off=None):
        q, k, v = self.parts
        return vp.vp_tokens(q=q.data_ptr() if self.queries else None, k=k.data_ptr(), v=v.data_ptr(),
                            q_stride=q.stride(0), k_stride=k.stride(0), v_stride=v.stride(0),
                            new_off=None if new_off is None else new_off.data_ptr(), n_tokens=self.n)


def rope(table, pos=None, sections=None, interleaved=False):
    """vp_rope of a device table [n_pos, rot] and positions int32 [axes, n]."""
    sec = list(sections or []) + [0] * (4 - len(sections or []))
    return vp.vp_rope(cos_sin=table.data_ptr(), n_pos=table.shape[0], rot_dim=table.shape[1], interleaved=int(interleaved),
                      n_axes=len(sections) if sections else 1, pos=None if pos is None else pos.data_ptr(),
                      section=(ctypes.c_int32 * 4)(*sec))


def assert_rounded(got, want, dtype, ctx=""):
    """got: want rounded to the type: half a step, and for bfloat16, rounded through
    float32, 2^-16 of it more. Results below the type's normal numbers: half their step."""
    half = 2.0 ** -8 * (1 + 2.0 ** -15) if dtype == "bf16" else 2.0 ** -24
    tiny = 2.0 ** -134 if dtype == "bf16" else 2.0 ** -150
    err = np.abs(got - want)
    assert np.all(err <= half * np.abs(want) + tiny), f"{ctx}: {np.max(err / (np.abs(want) + 1e-300)):.3g} relative"


def attention_bound(r, dtype, n, d, TG):
    """Bound of |out - reference| [T, Hq, d]: the scores are sums of d products (fp32 queries in
    three parts: 3 d, the two small parts, at most 2^-7 of the whole, first) in float32, each
    rounding at most half a step of the largest partial sum; scaling, exponential and
    normaliser as in the 16-bit call; the value sums' order; the output's rounding."""
    span = float(r.span.max()) if r.span.size else 0.0
    z = (2 * d + 2) * EPS * span + 4 * EPS * 1.45 * 2 * span
    e = 2 * z + 2 * (n / 32 + 32 + 16) * EPS + 8 * EPS
    e += 3 * (n / 32 + 32 + 16) * EPS  # (three parts of every weight)
    step = 2.0 ** -8 if dtype == "bf16" else EPS
    return e * r.spread + step * (np.abs(r.out) + e * r.spread) + 1e-37
