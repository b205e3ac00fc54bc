"""Layers that share lengths, segments and kept sets lose the same rows: vp_evict for each
layer's caches by one layer's sums, as the header says."""
import numpy as np
import pytest
import torch

from _parity import small_workload
from oracle import cache_oracle as CO
from paper_2605_31457_amd import step as S
from paper_2605_31457_amd import vp
from paper_2605_31457_amd import workloads as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,block", [("bf16", 0), ("f32", 16)])
def test_a_later_layer_follows_the_anchor(dtype, block):
    B, Hkv, budget = 2, 2, 96
    lens, segs = [200, 60], [[(5, 60), (100, 50)], [(9, 30)]]
    w = small_workload(5, B, 8, Hkv, 64, lens, segs, dtype=dtype, S_cap=256)
    later = small_workload(6, B, 8, Hkv, 64, lens, segs, dtype=dtype, S_cap=256)  # another layer's q, K and V
    ds, dl = S.DeviceStep(w, block_size=block), S.DeviceStep(later, block_size=block)
    dl.layout = ds.layout  # lengths, segments (and blocks) are shared
    ds.window_decode_attn(0, 4, sums=True)
    sums = ds.attn_sum.cpu().numpy()
    opt = vp.vp_evict_params(budget=budget, n_sink=4, n_recent=20)
    nbytes = vp.vp_evict_workspace_size(ds.shape, opt)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=ds.device)
    kept_later = torch.empty(B, budget, dtype=torch.int32, device=ds.device)
    new_len, seg_out = torch.full_like(ds.seq_len, -1), torch.full_like(ds.seg, -1)
    vp.vp_evict(dl.shape, ds.layout, opt, ds.attn_sum, dl.K, dl.V, kept_later, torch.empty_like(ds.attn_sum), seg_out,
                new_len, ws)
    assert ds.seq_len.tolist() == lens
    kept = ds.evict(budget, 4, 20)  # the last layer's call, in place
    assert torch.equal(kept, kept_later) and torch.equal(new_len, ds.seq_len) and torch.equal(seg_out, ds.seg)
    small = []
    for x in (w, later):
        K, V, lens2, segs2 = x.K.copy(), x.V.copy(), [], []
        for b, L in enumerate(lens):
            rows = CO.kept_rows(sums[b].astype(np.float64).sum(0).astype(np.float32), L, budget, 4, 20)
            K[b, :, :len(rows)], V[b, :, :len(rows)] = x.K[b][:, rows], x.V[b][:, rows]
            lens2.append(len(rows))
            segs2.append([s for s in CO.compact_segments(segs[b], rows) if s[1] > 0])
        c = W.Workload(name="compact", dtype=dtype, B=B, Hq=x.Hq, Hkv=Hkv, d=x.d, S_cap=x.S_cap,
                       seq_len=np.array(lens2, np.int32), segments=segs2, q=x.q, K=K, V=V, tau_mass=x.tau_mass,
                       r_lo_bp=x.r_lo_bp, r_hi_bp=x.r_hi_bp, clamp=x.clamp)
        small.append(S.DeviceStep(c, block_size=block, k_cap=ds.k_cap, max_vis=ds.max_vis))
    runs = []
    for anchor, layer in ((ds, dl), small):
        anchor.vis_idx.fill_(-7)
        anchor.decode_step()
        vp.vp_sparse_decode_attn(layer.shape, anchor.layout, layer.params, layer.q, layer.K, layer.V, anchor.vis_idx,
                                 anchor.k, layer.out, 0, layer.ws, layer.ws_bytes)
        torch.cuda.synchronize()
        runs.append((anchor.vis_idx, anchor.k, anchor.out, layer.out))
    for x, y in zip(*runs):
        assert torch.equal(x, y)
