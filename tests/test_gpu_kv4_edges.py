"""Attention over 4-bit caches: NaN blocks in tiles that every query sees whole, other streams in
order, shapes whose unused fields are zero."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from oracle import kv4_oracle as KO
from paper_2605_31457_amd import vp
from _cache import DEV, Caches, i32, rounded, torch_dtype
from _kv4 import Four, New, attention_bound, cos_sin, rope

pytestmark = pytest.mark.gpu


def _held(x):
    return KO.decode(*KO.quantise(x))


def _attention(c, q, lens, window=0, n_sink=0, scale=0.0, stream=None, shape=None):
    """One vp_kv4_decode_attn call on `stream`, ordered behind what the current one has made for it."""
    B, T, Hq, d = q.shape
    shape = shape or c.shape(Hq, "bf16" if q.dtype == torch.bfloat16 else "f32", T)
    w = vp.vp_window(window=window, n_sink=n_sink, sm_scale=scale)
    seq_len = i32(lens)
    out = torch.full_like(q, 7.0)
    nbytes = vp.vp_kv4_workspace_size(shape, w)
    ws = torch.full((nbytes + 64,), 0xff, dtype=torch.uint8, device=DEV)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    vp.vp_kv4_decode_attn(shape, c.layout(seq_len), w, q, c.struct(), out, ws, nbytes, stream)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0xff).all())
    return out


# ---------------------------------------------------------------------------
# NaN blocks
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 32])
@pytest.mark.parametrize("Hq,T,d", [(14, 1, 128), (14, 2, 128), (8, 1, 64), (8, 3, 64)])  # up to 8 query rows, and more
@pytest.mark.parametrize("L,window", [(400, 0), (1900, 0), (1900, 600)])  # one work-group, several
def test_nan_in_a_tile_that_all_see(L, window, Hq, T, d, page, dtype):
    """A block of 32 values that is NaN, of one row that every query sees whole tiles around: those elements of
    that KV head's outputs are NaN, and nothing else changes. Of a key: its KV head's outputs."""
    rng = np.random.default_rng(L + T)
    Hkv, B = 2, 2
    G = Hq // Hkv
    lens, cap = [L, 40], 416 if L == 400 else 2000
    c = Four(B, Hkv, cap, d, page=page, seed=2)
    c.put(*([rng.standard_normal((Hkv, n, d)) for n in lens] for _ in range(2)))
    qd = torch.from_numpy(rng.standard_normal((B, T, Hq, d))).to(torch_dtype(dtype)).to(DEV)
    ref = _attention(c, qd, lens, window, 4)
    assert bool(ref.isfinite().all())
    row = L - 200  # (tiles 100 rows before the queries and 100 behind a window's begin)
    at = (int(c.table[0, row // page]), row % page) if page else (0, row)
    k_scales, v_scales = c.scales
    old = int(v_scales[at[0], 1, at[1], 1])
    v_scales[at[0], 1, at[1], 1] = 255
    got = _attention(c, qd, lens, window, 4)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[0, :, G:, 32:64] = True
    assert bool((got.isnan() == bad).all()) and bool((got[~bad] == ref[~bad]).all())
    v_scales[at[0], 1, at[1], 1] = old
    k_scales[at[0], 0, at[1], 1] = 255
    got = _attention(c, qd, lens, window, 4)
    bad.zero_()
    bad[0, :, :G] = True
    assert bool((got.isnan() == bad).all()) and bool((got[~bad] == ref[~bad]).all())


# ---------------------------------------------------------------------------
# streams
# ---------------------------------------------------------------------------
def test_other_streams_in_order():
    """The same bits on another stream, behind the kernels that prepare the call's buffers."""
    rng = np.random.default_rng(11)
    lens, Hq, Hkv, d = [2100, 900, 1500], 28, 4, 128
    c = Four(3, Hkv, 2500, d, page=32, seed=1)
    K, V = ([rng.standard_normal((Hkv, n, d)) for n in lens] for _ in range(2))
    c.put(K, V)
    q = rounded(rng.standard_normal((3, 1, Hq, d)), "bf16")
    qd = torch.from_numpy(q).to(torch.bfloat16).to(DEV)
    ref = _attention(c, qd, lens)
    for b in range(3):
        r = CO.window_attention(q[b], _held(K[b]), _held(V[b]), 0, 0)
        assert np.all(np.abs(ref[b].double().cpu().numpy() - r.out) <= attention_bound(r, "bf16", lens[b], d, Hq)), b
    s = torch.cuda.Stream()
    for stream in (None, s, s, None):
        assert bool((_attention(c, qd, lens, stream=stream) == ref).all())


# ---------------------------------------------------------------------------
# fields of the shape that are not looked at
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 16])
def test_unused_fields_are_zero(page, dtype):
    rng = np.random.default_rng(page)
    lens, counts, Hq, Hkv, d = [70, 33], [70, 33], 8, 2, 64
    new = New(rng, sum(counts), Hq, Hkv, d, dtype)
    t = torch.from_numpy(cos_sin(80, d)).to(DEV)
    seq_len, off = i32(lens), i32([0, 70, 103])
    qd = torch.from_numpy(rng.standard_normal((2, 1, Hq, d))).to(torch_dtype(dtype)).to(DEV)
    runs = []
    for zeros in (False, True):
        four, wide = Four(2, Hkv, 80, d, page=page, seed=3), Caches(*np.zeros((2, 2, Hkv, 80, d)), dtype, page=page, seed=3)
        s4, s = four.shape(Hq, dtype), wide.shape(Hq)
        if zeros:
            s4.max_vis = s4.max_segs = s4.k_cap = s4.kv_stride_s = 0
            s.max_vis = s.max_segs = s.k_cap = 0
        q4, q = (torch.zeros(new.n, Hq, d, dtype=new.dev.dtype, device=DEV) for _ in range(2))
        vp.vp_append_kv4(s4, four.layout(seq_len), rope(t), new.struct(off), q4, four.struct())
        vp.vp_append_kv(s, wide.layout(seq_len), rope(t), new.struct(off), q, wide.K, wide.V)
        out4 = _attention(four, qd, lens, shape=s4)
        out = torch.zeros_like(qd)
        w = vp.vp_window(window=0, n_sink=0, sm_scale=0.0)
        n = vp.vp_window_workspace_size(s, w, False)
        ws = torch.zeros(max(n, 1), dtype=torch.uint8, device=DEV)
        vp.vp_window_decode_attn(s, wide.layout(seq_len), w, qd, wide.K, wide.V, None, out, ws, n)
        K, V = (torch.zeros_like(x) for x in (wide.K, wide.V))
        read = Caches.__new__(Caches)
        read.table = four.table  # (the 4-bit cache's blocks)
        vp.vp_kv4_read(s, read.layout(seq_len), four.struct(), None, K, V)
        torch.cuda.synchronize()
        runs.append([*four.codes, *four.scales, wide.K, wide.V, q4, q, out4, out, K, V])
    for i, (a, b) in enumerate(zip(*runs)):
        assert torch.equal(a, b), i
    assert all(bool(x.any()) for x in runs[1])
