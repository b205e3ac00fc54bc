"""How window attention splits its work, as far as the workspace shows it (no GPU): walks
that are shared out need room for their parts, one work-group per pair none."""
import pytest

from paper_2605_31457_amd import vp


def size(B, Hkv, cap, window, n_sink=0, sums=False, dtype=vp.VP_BF16, d=128, T=1):
    s = vp.vp_shape(batch=B, n_q_heads=4 * Hkv, n_kv_heads=Hkv, head_dim=d, dtype=dtype, max_seq_len=cap, max_vis=1,
                    max_segs=0, k_cap=1, block_size=0, scope=0, n_queries=T, kv_stride_b=Hkv * cap * d,
                    kv_stride_h=cap * d, kv_stride_s=d)
    return vp.vp_window_workspace_size(s, vp.vp_window(window=window, n_sink=n_sink, sm_scale=0.0), sums)


@pytest.mark.parametrize("sums", [False, True])
@pytest.mark.parametrize("dtype,d", [(vp.VP_BF16, 128), (vp.VP_BF16, 64), (vp.VP_F32, 64)])
@pytest.mark.parametrize("B,Hkv,cap", [(1, 4, 9000), (24, 8, 32768), (64, 4, 32768), (64, 8, 4096), (128, 8, 32768),
                                       (300, 4, 2048)])
def test_a_window_past_the_capacity_is_none(B, Hkv, cap, dtype, d, sums):
    """Lengths differ as much under a window that cuts nothing as without one."""
    for T in (1, 2):
        none = size(B, Hkv, cap, 0, 0, sums, dtype, d, T)
        for window, n_sink in ((cap, 0), (cap, 64), (cap + 1000, 4), (2 ** 31 - 1, 2 ** 31 - 1), (0, 64)):
            assert size(B, Hkv, cap, window, n_sink, sums, dtype, d, T) == none, (window, n_sink)


def test_long_walks_of_many_pairs_are_shared_out():
    """One full context among short ones must not leave its pairs to a work-group each."""
    assert size(128, 8, 32768, 0) > 0 and size(256, 4, 32768, 0) > 0 and size(64, 4, 32768, 32000) > 0
    assert size(512, 4, 32768, 0) > 0
    # (short beside what dealing costs: few tiles, or lengths of many sequences to read)
    assert size(128, 8, 1024, 0) == 0 and size(2048, 4, 32768, 0) == 0 and size(4096, 1, 32768, 0) == 0
    # both sides of the capacities in test_gpu_window_split.py
    for B, Hkv, d, whole, dealt in ((165, 2, 64, 69, 72), (40, 8, 64, 51, 54), (40, 8, 128, 51, 54), (50, 4, 64, 32, 35)):
        assert size(B, Hkv, 32 * whole, 0, d=d) == 0 and size(B, Hkv, 32 * dealt, 0, d=d) > 0
    assert size(64, 4, 32768, 8192) == 0  # (a window that cuts them)
