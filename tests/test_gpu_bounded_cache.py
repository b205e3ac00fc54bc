"""A decode loop on a bounded cache, as a serving program runs it: rows appended,
attention with running sums, eviction whenever the caches have grown, and the
method's decode step on what eviction leaves."""
import numpy as np
import pytest
import torch

from _cache import assert_attention, weight_error, EPS
from _parity import small_workload
from oracle import cache_oracle as CO
from oracle import vp_oracle as O
from paper_2605_31457_amd import step as S
from paper_2605_31457_amd import vp
from paper_2605_31457_amd import workloads as W

pytestmark = pytest.mark.gpu


def _stored(x, dtype):
    """x as it is stored, and as float64."""
    s = x.astype(np.float32) if dtype == "f32" else W.bf16_round(x.astype(np.float32))
    return s, O.as_f64(s)


@pytest.mark.parametrize("dtype,T,block,groups", [("bf16", 1, 0, False), ("bf16", 2, 16, False), ("f32", 1, 32, True),
                                                  ("bf16", 1, 0, True)])
def test_decode_loop(dtype, T, block, groups):
    B, Hq, Hkv, d, cap = 3, 8, 2, 64, 224
    budget, n_sink, n_recent, window = 128, 4, 24, 90
    lens = [150, 40, 97]
    segs = [[(5, 60)], [], [(20, 30), (60, 20)]] if not groups else [[]] * 3
    w = small_workload(31, B, Hq, Hkv, d, lens, segs, dtype=dtype, S_cap=cap)
    g = np.random.default_rng(7)
    if T > 1:
        w.q = np.repeat(w.q[:, None], T, 1)
    ds = S.DeviceStep(w, block_size=block, kv_groups=groups, max_vis=max(w.max_vis, 1))
    K, V = O.as_f64(w.K).copy(), O.as_f64(w.V).copy()
    want_s, bound_s = np.zeros((B, Hkv, cap)), np.zeros((B, Hkv, cap))
    view = lambda x: torch.from_numpy(x) if dtype == "f32" else torch.from_numpy(x.view(np.int16)).view(torch.bfloat16)

    def row(b, j):  # where row j of sequence b lies
        return (b, slice(None), j) if not block else (int(ds.block_table[b, j // block]), slice(None), j % block)

    evictions = 0
    for step in range(60):
        # T new rows per sequence, and their queries
        q, qf = _stored(g.standard_normal((B, T, Hq, d)), dtype)
        k, kf = _stored(0.5 * g.standard_normal((B, Hkv, T, d)), dtype)
        v, vf = _stored(0.5 * g.standard_normal((B, Hkv, T, d)), dtype)
        ds.q.copy_(view(q).view(ds.q.shape))
        for b in range(B):
            for t in range(T):
                j = lens[b] + t
                K[b, :, j], V[b, :, j] = kf[b, :, t], vf[b, :, t]
                ds.K[row(b, j)], ds.V[row(b, j)] = view(k[b, :, t].copy()).cuda(), view(v[b, :, t].copy()).cuda()
            lens[b] += T
        ds.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        # one window layer, one layer over everything that leaves its weights
        for win, sums in ((window, False), (0, True)):
            ds.window_decode_attn(win, n_sink, sums=sums)
            out = ds.out.view(B, T, Hq, d)
            for b, L in enumerate(lens):
                r = CO.window_attention(qf[b], K[b, :, :L], V[b, :, :L], win, n_sink)
                assert_attention(out[b], r, dtype, L, f"step {step} seq {b} window {win}")
                if sums:
                    new = slice(L - T, L)
                    want_s[b, :, new] = bound_s[b, :, new] = 0.0
                    want_s[b, :, :L] += r.weight
                    TG = T * Hq // Hkv
                    # this call's weights, and its additions' rounding
                    bound_s[b, :, :L] += (weight_error(r, d, L, TG) + (TG + 1) * EPS) * r.weight + EPS * want_s[b, :, :L]
        got_s = ds.attn_sum.cpu().numpy()
        for b, L in enumerate(lens):
            assert np.all(np.abs(got_s[b, :, :L] - want_s[b, :, :L]) <= bound_s[b, :, :L] + 1e-37), f"step {step} seq {b}"
        if max(lens) + T <= 160:
            continue
        evictions += 1
        kept = ds.evict(budget, n_sink, n_recent).cpu().numpy().reshape(B, -1, budget)
        after_s = ds.attn_sum.cpu().numpy()
        for b, L in enumerate(lens):
            for u in range(kept.shape[1]):
                score = got_s[b, u] if groups else got_s[b].astype(np.float64).sum(0).astype(np.float32)
                rows = CO.kept_rows(score, L, budget, n_sink, n_recent)
                n = len(rows)
                assert np.array_equal(kept[b, u, :n], rows) and np.all(kept[b, u, n:] == -1), f"step {step} seq {b}"
                for h in [u] if groups else range(Hkv):
                    for x in (K, V, want_s, bound_s):
                        x[b, h, :n] = x[b, h, rows]
                    assert np.array_equal(after_s[b, h, :n], got_s[b, h, rows])
            if not groups:
                segs[b] = CO.compact_segments(segs[b], rows)
            lens[b] = min(L, budget)
        assert ds.seq_len.tolist() == lens
        if not groups:
            flat = [list(s) for x in segs for s in x]
            assert ds.seg.view(-1, 2)[:len(flat)].tolist() == flat
            if T == 1:
                step_after_eviction(ds, w, dtype, K, V, qf, lens, segs, block)
    assert evictions >= 2


def step_after_eviction(ds, w, dtype, K, V, qf, lens, segs, block):
    """The method's step on the evicted caches gives what it gives on caches that
    never held more (segments that lost all their rows left out)."""
    ds.vis_idx.fill_(-7)
    ds.decode_step()
    got = ds.results()
    Ks, Vs = _stored(K, dtype)[0], _stored(V, dtype)[0]
    w2 = W.Workload(name="compact", dtype=dtype, B=w.B, Hq=w.Hq, Hkv=w.Hkv, d=w.d, S_cap=w.S_cap,
                    seq_len=np.array(lens, np.int32), segments=[[s for s in x if s[1] > 0] for x in segs],
                    q=_stored(qf[:, 0], dtype)[0], K=Ks, V=Vs, tau_mass=w.tau_mass, r_lo_bp=w.r_lo_bp,
                    r_hi_bp=w.r_hi_bp, clamp=w.clamp)
    d2 = S.DeviceStep(w2, block_size=block, k_cap=ds.k_cap, max_vis=ds.max_vis)
    d2.decode_step()
    want = d2.results()
    for key in ("mass_head", "mass_seq", "k", "vis_idx", "out"):
        assert np.array_equal(got[key], want[key]), key
    for b, x in enumerate(segs):
        n = sum(s[1] for s in x)
        assert np.array_equal(got["scores"][b, :n], want["scores"][b, :n])
    ds.out.zero_()


def test_loop_captured_in_graphs():
    """One graph of the attention with sums and one of the eviction, replayed in turn
    with eager work between, against the same calls made eagerly."""
    w = small_workload(5, 2, 8, 2, 64, [200, 170], [[(5, 60)], [(9, 40)]], S_cap=256)
    runs = []
    for captured in (False, True):
        ds = S.DeviceStep(w)
        ds.window_decode_attn(0, 4, sums=True)  # (allocates)
        ds.attn_sum.zero_()
        torch.cuda.synchronize()
        attend = lambda: ds.window_decode_attn(0, 4, sums=True)
        kept = torch.zeros(2, 128, dtype=torch.int32, device=ds.device)
        opt = vp.vp_evict_params(budget=128, n_sink=4, n_recent=32)
        ws = torch.empty(vp.vp_evict_workspace_size(ds.shape, opt), dtype=torch.uint8, device=ds.device)
        evict = lambda: vp.vp_evict(ds.shape, ds.layout, opt, ds.attn_sum, ds.K, ds.V, kept, ds.attn_sum, ds.seg,
                                    ds.seq_len, ws)
        if captured:
            graphs = []
            for f in (attend, evict):
                graphs.append(torch.cuda.CUDAGraph())
                with torch.cuda.graph(graphs[-1]):
                    f()
            attend, evict = graphs[0].replay, graphs[1].replay
        log = []
        for rep in range(3):
            for _ in range(3):
                attend()
                torch.cuda.synchronize()
                log.append(ds.out.clone())
                ds.q.mul_(0.5 if rep % 2 else 2.0)
            evict()
            log += [x.clone() for x in (kept, ds.attn_sum, ds.K, ds.V, ds.seq_len, ds.seg)]
            ds.seq_len.add_(60)  # (as if 60 rows had been appended)
        torch.cuda.synchronize()
        runs.append(log)
    for i, (x, y) in enumerate(zip(*runs)):
        assert torch.equal(x, y), i


def test_evict_needs_sums():
    ds = S.DeviceStep(small_workload(5, 1, 4, 1, 64, [50], [[]]))
    with pytest.raises(RuntimeError):
        ds.evict(10)


@pytest.mark.parametrize("handle", [False, True])
def test_buffers_made_on_the_calls_own_stream(handle):
    """The first call on a side stream while the current stream is busy: attn_sum is
    cleared before the call adds to it, and the rows kept are not given away while
    the call runs."""
    w = small_workload(5, 2, 8, 2, 64, [200, 170], [[(5, 60)], [(9, 40)]], S_cap=256)
    runs = []
    for side in (None, torch.cuda.Stream()):
        ds = S.DeviceStep(w)
        busy = torch.zeros(1 << 28, dtype=torch.float32, device=ds.device)
        torch.cuda.synchronize()
        stream = side.cuda_stream if handle and side is not None else side
        for _ in range(20 if side is not None else 0):
            busy.add_(1.0)  # (0.5 ms each, on the current stream)
        ds.window_decode_attn(0, 4, sums=True, stream=stream)
        kept = ds.evict(128, 4, 32, stream=stream)
        torch.cuda.synchronize()
        runs.append([kept, ds.attn_sum, ds.out, ds.K, ds.seq_len])
    for x, y in zip(*runs):
        assert torch.equal(x, y)
    assert float(runs[1][1].sum()) > 0
