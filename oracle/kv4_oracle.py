"""fp64 reference of the calls that fill caches and of 4-bit rows (vp_append_kv,
vp_append_kv4, vp_kv4_read).

TEST INFRASTRUCTURE, like vp_oracle: the definitions written out in float64, without
code shared with the library. Attention over 4-bit rows is cache_oracle's on the values
that the rows hold.
"""
from __future__ import annotations

import numpy as np

__all__ = ["rotate", "axis_of_pairs", "quantise", "decode", "VALUES"]

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])  # by the three low bits of a code
SCALE_MIN, SCALE_MAX, SCALE_NAN = 2, 252, 255


def axis_of_pairs(rot, sections):
    """The axis of every pair; sections None: one axis."""
    if sections is None:
        return np.zeros(rot // 2, np.int64)
    return np.repeat(np.arange(len(sections)), sections)


def rotate(x, cos_sin, pos, rot, sections=None, interleaved=False):
    """x [n, H, d]; cos_sin [n_pos, rot] as stored; pos [axes, n]. float64 [n, H, d]."""
    x = np.asarray(x, np.float64)
    if rot == 0:
        return x.copy()
    table = np.asarray(cos_sin, np.float64)
    axis = axis_of_pairs(rot, sections)
    out = x.copy()
    for i in range(rot // 2):
        p = np.clip(np.asarray(pos)[axis[i]], 0, table.shape[0] - 1)
        c, s = table[p, i][:, None], table[p, rot // 2 + i][:, None]
        u, v = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        out[..., u] = x[..., u] * c - x[..., v] * s
        out[..., v] = x[..., v] * c + x[..., u] * s
    return out


def quantise(x):
    """x [..., d] -> (codes uint8 [..., d], scale bytes uint8 [..., d / 32])."""
    x = np.asarray(x, np.float64)
    y = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(y).max(-1)
    bad = ~np.isfinite(y).all(-1)
    scale = np.full(top.shape, 2.0 ** -125)
    byte = np.full(top.shape, SCALE_MIN, np.int64)
    for e in range(-125, 125):
        # (one step up wherever this power of two is too small)
        small = top > 7.0 * 2.0 ** e
        scale[small] = 2.0 ** (e + 1)
        byte[small] = e + 1 + 127
    with np.errstate(invalid="ignore"):
        a = np.abs(y) / scale[..., None]
    code = np.zeros(a.shape, np.uint8)
    for i in range(7):
        mid = (VALUES[i] + VALUES[i + 1]) / 2
        up = a >= mid if (i + 1) % 2 == 0 else a > mid  # a tie goes to the even code
        code[up] = i + 1
    code |= (np.signbit(y).astype(np.uint8) << 3)
    code[bad] = 0
    byte[bad] = SCALE_NAN
    return code.reshape(x.shape), byte.astype(np.uint8)


def decode(code, byte):
    """The values, float64; NaN in blocks marked so."""
    code = np.asarray(code)
    v = np.where(code & 8, -1.0, 1.0) * VALUES[code & 7]
    s = np.where(np.asarray(byte) == SCALE_NAN, np.nan, 2.0 ** (np.asarray(byte, np.float64) - 127))
    return (v.reshape(*byte.shape, 32) * s[..., None]).reshape(code.shape)
