"""vp_append_kv: rotation and the rows written, against the reference."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as KO
from paper_2605_31457_amd import vp
from _cache import DEV, Caches, i32, rounded
from _kv4 import New, assert_rounded, cos_sin, rope

pytestmark = pytest.mark.gpu


def _append(c, new, lens, Hq, T=1, new_off=None, r=None, q_out=None, stream=None):
    """One call; returns q_out."""
    if q_out is None and new.queries:
        q_out = torch.full((new.n, Hq, c.K.shape[3]), 7.0, dtype=new.dev.dtype, device=DEV)
    off = None if new_off is None else i32(new_off)
    seq_len = i32(lens)
    vp.vp_append_kv(c.shape(Hq, T), c.layout(seq_len), r, new.struct(off), q_out, c.K, c.V, stream)
    torch.cuda.synchronize()
    return q_out


def _check(c, new, lens, counts, K0, V0, rot, pos, table, sections, interleaved, q_out, ctx=""):
    """Rows of every sequence: the new tokens last, everything else as before."""
    K, V = c.get()
    kr = KO.rotate(new.k, table, pos, rot, sections, interleaved)
    qr = KO.rotate(new.q, table, pos, rot, sections, interleaved)
    i = 0
    for b, (L, n) in enumerate(zip(lens, counts)):
        L = min(max(L, 0), c.cap)
        out = max(0, n - L)  # tokens before row 0
        if q_out is not None:
            q = q_out.double().cpu().numpy()
            assert np.all(q[i:i + out] == 7.0), ctx
            assert_rounded(q[i + out:i + n], qr[i + out:i + n], new.dtype, ctx + " q")
        for got, old, want in ((K[b], K0[b], kr), (V[b], V0[b], new.v)):
            assert_rounded(got[:, L - n + out:L], want[i + out:i + n].transpose(1, 0, 2), new.dtype, ctx)
            assert np.array_equal(got[:, :L - n + out], old[:, :L - n + out]), ctx
            assert np.array_equal(got[:, L:], old[:, L:]), ctx
        i += n
    if q_out is not None:
        assert bool((q_out[i:] == 7.0).all()), ctx


def _caches(rng, B, Hkv, cap, d, dtype, **kw):
    K0, V0 = (rounded(rng.standard_normal((B, Hkv, cap, d)), dtype) for _ in range(2))
    return Caches(K0, V0, dtype, **kw), K0, V0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,rot", [(28, 4, 128, 128), (4, 1, 64, 64), (16, 16, 64, 32), (8, 8, 128, 16), (3, 3, 128, 112)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_steps(dtype, Hq, Hkv, d, rot, interleaved):
    """Decode steps: one token per sequence at its row's position."""
    rng = np.random.default_rng(rot + Hq)
    lens = [1, 17, 33, 40]
    c, K0, V0 = _caches(rng, 4, Hkv, 40, d, dtype)
    new = New(rng, 4, Hq, Hkv, d, dtype)
    table = cos_sin(64, rot)
    t = torch.from_numpy(table).to(DEV)
    q = _append(c, new, lens, Hq, r=rope(t, interleaved=interleaved))
    pos = np.array([[L - 1 for L in lens]])
    _check(c, new, lens, [1] * 4, K0, V0, rot, pos, table, None, interleaved, q)


@pytest.mark.parametrize("order,page", [("bhs", 0), ("bsh", 0), ("pad", 0), ("bhs", 1), ("bhs", 8), ("bsh", 32), ("pad", 64)])
@pytest.mark.parametrize("dtype,fused", [("bf16", True), ("f32", False)])
def test_ragged_chunks(order, page, dtype, fused):
    """Ragged chunks with sequences that get nothing, strides and pages; positions that are not the
    rows, some outside the table; rows of q, k, v past the last sequence."""
    rng = np.random.default_rng(page + 5)
    lens, counts = [70, 5, 0, 33, 64, 9], [37, 5, 0, 0, 64, 1]
    Hq, Hkv, d, rot = 8, 2, 128, 128
    c, K0, V0 = _caches(rng, 6, Hkv, 80, d, dtype, order=order, page=page, seed=page)
    n = sum(counts)
    new = New(rng, n + 3, Hq, Hkv, d, dtype, fused=fused)
    table = cos_sin(100, rot, 1)
    t = torch.from_numpy(table).to(DEV)
    pos = rng.integers(-20, 130, (1, n + 3))
    off = np.concatenate([[0], np.cumsum(counts)])
    p = i32(pos.tolist())
    q = _append(c, new, lens, Hq, new_off=off.tolist(), r=rope(t, p))
    _check(c, new, lens, counts, K0, V0, rot, pos, table, None, False, q)


@pytest.mark.parametrize("d,rot,sections", [(128, 128, (16, 24, 24)), (128, 64, (8, 12, 12)), (64, 64, (4, 0, 20, 8)), (128, 128, (60, 4))])
@pytest.mark.parametrize("interleaved", [False, True])
def test_axes(d, rot, sections, interleaved):
    rng = np.random.default_rng(rot + len(sections))
    lens, counts, Hq, Hkv = [21, 50], [20, 11], 4, 2
    c, K0, V0 = _caches(rng, 2, Hkv, 50, d, "bf16")
    new = New(rng, 31, Hq, Hkv, d, "bf16")
    table = cos_sin(64, rot, 2)
    t = torch.from_numpy(table).to(DEV)
    pos = rng.integers(0, 64, (len(sections), 31))
    p = i32(pos.tolist())
    q = _append(c, new, lens, Hq, new_off=[0, 20, 31], r=rope(t, p, sections, interleaved))
    _check(c, new, lens, counts, K0, V0, rot, pos, table, sections, interleaved, q)


def test_no_rotation_no_queries():
    rng = np.random.default_rng(1)
    lens, counts, Hq, Hkv, d = [6, 30], [4, 25], 12, 3, 64
    for dtype in ("bf16", "f32"):
        c, K0, V0 = _caches(rng, 2, Hkv, 31, d, dtype)
        new = New(rng, 29, Hq, Hkv, d, dtype, queries=False)
        _append(c, new, lens, Hq, new_off=[0, 4, 29])
        _check(c, new, lens, counts, K0, V0, 0, None, None, None, False, None)


def test_sequences_shorter_than_their_tokens():
    """Their first tokens have no row: left out, their queries too. Lengths outside the capacity are clipped."""
    rng = np.random.default_rng(2)
    lens, Hq, Hkv, d = [3, 0, 1, 90, -4], 4, 2, 64
    c, K0, V0 = _caches(rng, 5, Hkv, 40, d, "bf16")
    new = New(rng, 20, Hq, Hkv, d, "bf16")
    table = cos_sin(64, 64)
    t = torch.from_numpy(table).to(DEV)
    pos = np.concatenate([np.arange(min(max(L, 0), 40) - 4, min(max(L, 0), 40)) for L in lens])[None]
    q = _append(c, new, lens, Hq, T=4, r=rope(t))
    _check(c, new, lens, [4] * 5, K0, V0, 64, pos, table, None, False, q)


def test_many_sequences():
    """More sequences than a wave probes at a time, most of them without tokens."""
    rng = np.random.default_rng(3)
    B, Hq, Hkv, d, cap = 4133, 2, 1, 64, 9
    counts = rng.integers(0, 3, B) * (rng.random(B) < 0.3)
    counts[[0, 63, 64, B - 1]] = 1
    lens = np.minimum(counts + rng.integers(0, 6, B), cap)
    c, K0, V0 = _caches(rng, B, Hkv, cap, d, "bf16")
    n = int(counts.sum())
    new = New(rng, n, Hq, Hkv, d, "bf16")
    table = cos_sin(16, 64)
    t = torch.from_numpy(table).to(DEV)
    off = np.concatenate([[0], np.cumsum(counts)])
    pos = np.concatenate([np.arange(L - m, L) for L, m in zip(lens, counts)])[None]
    q = _append(c, new, lens.tolist(), Hq, new_off=off.tolist(), r=rope(t))
    _check(c, new, lens.tolist(), counts.tolist(), K0, V0, 64, pos, table, None, False, q)


def test_in_place_and_large_chunks():
    """q_out = q; so many tokens that a wave takes all rows of one."""
    rng = np.random.default_rng(4)
    n, Hq, Hkv, d = 9001, 6, 2, 128
    c, K0, V0 = _caches(rng, 1, Hkv, 9100, d, "bf16", page=128)
    new = New(rng, n, Hq, Hkv, d, "bf16", fused=False)
    table = cos_sin(9100, 128)
    t = torch.from_numpy(table).to(DEV)
    q = _append(c, new, [9050], Hq, new_off=[0, n], r=rope(t), q_out=new.parts[0])
    pos = np.arange(9050 - n, 9050)[None]
    _check(c, new, [9050], [n], K0, V0, 128, pos, table, None, False, q)


def test_rounded_once():
    """Where the two products nearly cancel the result is still the 64-bit one rounded: nothing of it is
    lost to a product's own rounding."""
    n, d = 256, 64
    rng = np.random.default_rng(6)
    x = rounded(np.full((n, 3, d), 1.0), "f32")
    table = np.zeros((n, 64), np.float32)
    table[:, :32] = rng.uniform(0.5, 1, (n, 32))
    table[:, 32:] = np.nextafter(table[:, :32], np.float32(2))
    x[:, :, 32:] = rounded(rng.uniform(1 - 2e-7, 1 + 2e-7, (n, 3, 32)), "f32")
    c, K0, V0 = _caches(rng, 1, 1, n, d, "f32")
    new = New.__new__(New)
    new.set(x, 1, 1, "f32")
    t = torch.from_numpy(table).to(DEV)
    q = _append(c, new, [n], 1, new_off=[0, n], r=rope(t))
    _check(c, new, [n], [n], K0, V0, 64, np.arange(n)[None], table, None, False, q)


def test_far_rows():
    """Cache offsets beyond 32 bits: rows of a cache of 5 GB and of a block far into a pool."""
    rng = np.random.default_rng(7)
    Hkv, d, cap = 2, 128, 5 << 21  # 2.7 GB per head
    K = torch.zeros(1, Hkv, cap, d, dtype=torch.bfloat16, device=DEV)
    V = torch.zeros(1, Hkv, cap, d, dtype=torch.bfloat16, device=DEV)
    new = New(rng, 3, 2, Hkv, d, "bf16", queries=False)
    shape = vp.vp_shape(batch=1, n_q_heads=2, n_kv_heads=Hkv, head_dim=d, dtype=vp.VP_BF16, max_seq_len=cap, max_vis=1,
                        max_segs=1, k_cap=1, block_size=0, scope=0, n_queries=3, kv_stride_b=K.stride(0),
                        kv_stride_h=K.stride(1), kv_stride_s=d)
    L = i32([cap - 5])
    vp.vp_append_kv(shape, vp.vp_layout(seq_len=L.data_ptr(), vis_seg_off=None, vis_seg=None, block_table=None), None,
                    new.struct(), None, K, V)
    torch.cuda.synchronize()
    for x, want in ((K, new.k), (V, new.v)):
        assert np.array_equal(x[0, :, cap - 8:cap - 5].double().cpu().numpy(), want.transpose(1, 0, 2))
        assert not bool(x[0, :, cap - 5:].any()) and not bool(x[0, :, cap - 200:cap - 8].any())
    del K, V, x
    torch.cuda.empty_cache()


def test_stream_and_graph():
    """On another stream, and replayed with other tokens and lengths."""
    rng = np.random.default_rng(8)
    Hq, Hkv, d, B = 4, 2, 64, 3
    c, K0, V0 = _caches(rng, B, Hkv, 64, d, "bf16", page=16)
    new = New(rng, B, Hq, Hkv, d, "bf16")
    table = cos_sin(64, 64)
    t = torch.from_numpy(table).to(DEV)
    seq_len = i32([5, 16, 30])
    q_out = torch.zeros(B, Hq, d, dtype=torch.bfloat16, device=DEV)
    s = torch.cuda.Stream()
    args = (c.shape(Hq), c.layout(seq_len), rope(t), new.struct(), q_out, c.K, c.V)
    torch.cuda.synchronize()
    vp.vp_append_kv(*args, s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        vp.vp_append_kv(*args)
    lens = [5, 16, 30]
    for i in range(4):
        lens = [L + 1 for L in lens]
        seq_len.copy_(i32(lens))
        fresh = New(rng, B, Hq, Hkv, d, "bf16")
        new.dev.copy_(fresh.dev)
        K1, V1 = c.get()
        q_out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        _check(c, fresh, lens, [1] * B, K1, V1, 64, np.array([[L - 1 for L in lens]]), table, None, False, q_out)
