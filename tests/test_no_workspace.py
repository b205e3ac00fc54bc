"""The bounded-cache calls of the binding without a workspace (no GPU): what a call that needs
none takes, and the library's own refusal where it needs one."""
import pytest

from paper_2605_31457_amd import vp

PTR = 1 << 20  # an aligned address that nothing dereferences


def _shape():
    return vp.vp_shape(batch=2, n_q_heads=28, n_kv_heads=4, head_dim=128, dtype=vp.VP_BF16, max_seq_len=4096, max_vis=1,
                       max_segs=1, k_cap=1, block_size=0, kv_stride_b=4 * 4096 * 128, kv_stride_h=4096 * 128,
                       kv_stride_s=128)


def test_none_is_no_room():
    layout = vp.vp_layout(seq_len=PTR, vis_seg_off=None, vis_seg=None, block_table=None)
    w = vp.vp_window(window=0, n_sink=0, sm_scale=0.0)
    assert vp.vp_window_workspace_size(_shape(), w) > 0
    with pytest.raises(vp.VPError, match="VP_ERR_WORKSPACE"):
        vp.vp_window_decode_attn(_shape(), layout, w, PTR, PTR, PTR, None, PTR, None, stream=0)
    with pytest.raises(vp.VPError, match="VP_ERR_WORKSPACE"):
        vp.vp_evict(_shape(), layout, vp.vp_evict_params(budget=64, n_sink=0, n_recent=0), PTR, PTR, 2 * PTR, PTR, PTR,
                    None, PTR, None, stream=0)
