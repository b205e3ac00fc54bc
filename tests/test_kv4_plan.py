"""How attention over 4 bits splits its work, as far as the workspace shows it (no GPU): walks that are
dealt need room for their parts, one work-group per pair none."""
import pytest

from paper_2605_31457_amd import vp


def whole(B, Hkv, cap, window=0, n_sink=0, T=1, dtype=vp.VP_BF16, d=128):
    s = vp.vp_shape(batch=B, n_q_heads=4 * Hkv, n_kv_heads=Hkv, head_dim=d, dtype=dtype, max_seq_len=cap, n_queries=T)
    return vp.vp_kv4_workspace_size(s, vp.vp_window(window=window, n_sink=n_sink, sm_scale=0.0)) == 0


@pytest.mark.parametrize("dtype,d", [(vp.VP_BF16, 128), (vp.VP_BF16, 64), (vp.VP_F32, 128)])
def test_both_sides_of_the_rule(dtype, d):
    w = lambda *a, **kw: whole(*a, dtype=dtype, d=d, **kw)
    # short walks
    assert w(1, 4, 28 * 32) and not w(1, 4, 28 * 32 + 1) and w(1, 1, 1)
    # short beside what dealing costs: 1200 tiles up to pairs (350 + sequences)
    assert w(64, 4, 88 * 32) and not w(64, 4, 88 * 32 + 1)
    assert w(1024, 4, 32768) and not w(128, 4, 32768)
    # windows of up to half the capacity that nearly fill the CUs
    assert w(48, 4, 32768, window=8192) and not w(47, 4, 32768, window=8192)
    assert w(64, 4, 32768, window=8192, n_sink=64, T=2) and not w(64, 4, 32768, window=20000)
    # more tiles than the deal counts
    assert w(4096, 64, 1 << 20)


def test_a_window_past_the_capacity_is_none():
    for B, cap in ((1, 9000), (64, 32768), (128, 4096)):
        for window, n_sink in ((cap, 0), (cap + 1000, 4), (2 ** 31 - 1, 2 ** 31 - 1), (0, 64)):
            assert whole(B, 4, cap, window, n_sink) == whole(B, 4, cap)
