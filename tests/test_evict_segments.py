"""Eviction and visual segments: rows that every KV head keeps for itself have no common
positions, so sequences with visual tokens are evicted with one kept set."""
import pytest
import torch

from _parity import small_workload
from paper_2605_31457_amd import step as S


def test_segments_that_would_differ_by_head_are_refused():
    for segs, refused in (([[(5, 20)], []], True), ([[], []], False), ([[(5, 0)], []], False)):
        ds = S.DeviceStep(small_workload(5, 2, 8, 2, 64, [50, 40], segs), device="cpu", kv_groups=True, max_vis=64)
        ds.attn_sum = torch.zeros(2, 2, ds.w.S_cap)
        before = [x.clone() for x in (ds.K, ds.V, ds.seq_len, ds.seg)]
        # (a budget of none is refused by the library, before anything else happens)
        with pytest.raises(RuntimeError, match="differ by head" if refused else "VP_ERR_RANGE"):
            ds.evict(0 if not refused else 16, 1, 2)
        with pytest.raises(RuntimeError, match="VP_ERR_RANGE"):
            ds.evict(0, kv_groups=False)
        assert all(torch.equal(x, y) for x, y in zip(before, (ds.K, ds.V, ds.seq_len, ds.seg)))
    ds = S.DeviceStep(small_workload(5, 2, 8, 2, 64, [50, 40], [[(5, 20)], []]), device="cpu")
    ds.attn_sum = torch.zeros(2, 2, ds.w.S_cap)
    with pytest.raises(RuntimeError, match="differ by head"):
        ds.evict(16, 1, 2, kv_groups=True)
