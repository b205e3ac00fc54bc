"""Host side of the bounded-cache calls (no GPU): refusals before anything is
enqueued, workspace sizes, the walk over the rows, and the reference itself."""
import ctypes
import math

import numpy as np
import pytest

from oracle import cache_oracle as CO
from paper_2605_31457_amd import vp

PTR = 1 << 20  # an aligned address that nothing dereferences


def _shape(**kw):
    s = dict(batch=2, n_q_heads=28, n_kv_heads=4, head_dim=128, dtype=vp.VP_BF16, max_seq_len=4096, max_vis=1296,
             max_segs=1, k_cap=64, block_size=0, kv_stride_b=4 * 4096 * 128, kv_stride_h=4096 * 128, kv_stride_s=128)
    s.update(kw)
    return vp.vp_shape(**s)


def _layout(**kw):
    l = dict(seq_len=PTR, vis_seg_off=None, vis_seg=None, block_table=None)
    l.update(kw)
    return vp.vp_layout(**l)


def _window(**kw):
    return vp.vp_window(**dict(dict(window=1024, n_sink=4, sm_scale=0.0), **kw))


def _evict(**kw):
    return vp.vp_evict_params(**dict(dict(budget=2048, n_sink=4, n_recent=64), **kw))


def test_struct_sizes():
    assert ctypes.sizeof(vp.vp_window) == 12 and ctypes.sizeof(vp.vp_evict_params) == 12


@pytest.mark.parametrize("kw,status", [
    (dict(window=-1), "VP_ERR_RANGE"), (dict(n_sink=-1), "VP_ERR_RANGE"),
    (dict(sm_scale=math.nan), "VP_ERR_RANGE"), (dict(sm_scale=math.inf), "VP_ERR_RANGE"),
])
def test_window_options(kw, status):
    with pytest.raises(vp.VPError) as e:
        vp.vp_window_workspace_size(_shape(), _window(**kw))
    assert status in str(e.value)
    with pytest.raises(vp.VPError) as e:
        vp.vp_window_decode_attn(_shape(), _layout(), _window(**kw), PTR, PTR, PTR, None, PTR, PTR, 1 << 40, 0)
    assert status in str(e.value)


@pytest.mark.parametrize("kw,status", [
    (dict(budget=0), "VP_ERR_RANGE"), (dict(budget=-7), "VP_ERR_RANGE"), (dict(budget=(1 << 28) + 1), "VP_ERR_RANGE"),
    (dict(n_sink=-1), "VP_ERR_RANGE"), (dict(n_recent=-1), "VP_ERR_RANGE"),
    (dict(n_sink=2000, n_recent=49), "VP_ERR_RANGE"),
    (dict(n_sink=2 ** 31 - 1, n_recent=2 ** 31 - 1), "VP_ERR_RANGE"),
])
def test_evict_options(kw, status):
    with pytest.raises(vp.VPError) as e:
        vp.vp_evict_workspace_size(_shape(), _evict(**kw))
    assert status in str(e.value)


def _call_window(shape=None, layout=None, q=PTR, K=PTR, V=PTR, sums=None, out=PTR, ws=PTR, nbytes=1 << 40):
    vp.vp_window_decode_attn(shape or _shape(), layout or _layout(), _window(), q, K, V, sums, out, ws, nbytes, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), "VP_ERR_NULL"), (dict(K=None), "VP_ERR_NULL"), (dict(V=None), "VP_ERR_NULL"),
    (dict(out=None), "VP_ERR_NULL"), (dict(layout=_layout(seq_len=None)), "VP_ERR_NULL"),
    (dict(shape=_shape(block_size=32)), "VP_ERR_NULL"),  # paged, no block table
    (dict(q=PTR + 8), "VP_ERR_SHAPE"), (dict(K=PTR + 2), "VP_ERR_SHAPE"), (dict(V=PTR + 4), "VP_ERR_SHAPE"),
    (dict(out=PTR + 8), "VP_ERR_SHAPE"), (dict(sums=PTR + 2), "VP_ERR_SHAPE"),
    (dict(ws=None), "VP_ERR_WORKSPACE"), (dict(ws=PTR + 16), "VP_ERR_WORKSPACE"), (dict(nbytes=100), "VP_ERR_WORKSPACE"),
    (dict(shape=_shape(head_dim=96)), "VP_ERR_UNSUPPORTED"), (dict(shape=_shape(dtype=3)), "VP_ERR_DTYPE"),
    (dict(shape=_shape(n_queries=3)), "VP_ERR_UNSUPPORTED"), (dict(shape=_shape(kv_stride_s=130)), "VP_ERR_SHAPE"),
])
def test_window_refusals(kw, status):
    with pytest.raises(vp.VPError) as e:
        _call_window(**kw)
    assert status in str(e.value)


def _call_evict(shape=None, layout=None, sums=PTR, K=PTR, V=2 * PTR, kept=PTR, out=PTR, seg=None, new_len=PTR, ws=PTR,
                nbytes=1 << 40):
    vp.vp_evict(shape or _shape(), layout or _layout(), _evict(), sums, K, V, kept, out, seg, new_len, ws, nbytes, 0)


@pytest.mark.parametrize("kw,status", [
    (dict(sums=None), "VP_ERR_NULL"), (dict(K=None), "VP_ERR_NULL"), (dict(V=None), "VP_ERR_NULL"),
    (dict(kept=None), "VP_ERR_NULL"), (dict(out=None), "VP_ERR_NULL"), (dict(new_len=None), "VP_ERR_NULL"),
    (dict(layout=_layout(seq_len=None)), "VP_ERR_NULL"), (dict(shape=_shape(block_size=16)), "VP_ERR_NULL"),
    (dict(seg=PTR), "VP_ERR_NULL"),  # segments wanted, none in the layout
    (dict(seg=PTR, layout=_layout(vis_seg_off=PTR, vis_seg=PTR), shape=_shape(scope=1)), "VP_ERR_UNSUPPORTED"),
    (dict(K=PTR + 8), "VP_ERR_SHAPE"), (dict(V=2 * PTR + 8), "VP_ERR_SHAPE"), (dict(V=PTR), "VP_ERR_SHAPE"),
    (dict(ws=None), "VP_ERR_WORKSPACE"), (dict(ws=PTR + 64), "VP_ERR_WORKSPACE"), (dict(nbytes=8), "VP_ERR_WORKSPACE"),
    # caches whose rows share memory: one head or one sequence for all, heads too close, blocks too close
    (dict(shape=_shape(kv_stride_h=0)), "VP_ERR_SHAPE"), (dict(shape=_shape(kv_stride_b=0)), "VP_ERR_SHAPE"),
    (dict(shape=_shape(kv_stride_h=2048 * 128)), "VP_ERR_SHAPE"),
    (dict(shape=_shape(block_size=32, kv_stride_h=32 * 128, kv_stride_b=3 * 32 * 128), layout=_layout(block_table=PTR)),
     "VP_ERR_SHAPE"),
    (dict(shape=_shape(head_dim=80)), "VP_ERR_UNSUPPORTED"), (dict(shape=_shape(max_seq_len=0)), "VP_ERR_SHAPE"),
])
def test_evict_refusals(kw, status):
    with pytest.raises(vp.VPError) as e:
        _call_evict(**kw)
    assert status in str(e.value)


def test_sum_workspace_holds_the_logits():
    w = _window(window=0)
    plain, sums = (vp.vp_window_workspace_size(_shape(), w, s) for s in (False, True))
    assert sums - plain >= 2 * 4 * 4096 * 7 * 4  # [B][Hkv][rows][G] float
    # a window bounds it, whatever the cache's capacity
    a = vp.vp_window_workspace_size(_shape(max_seq_len=1 << 20), _window(), True)
    assert a <= vp.vp_window_workspace_size(_shape(max_seq_len=1 << 27), _window(), True) + 256 <= 2 * a
    with pytest.raises(vp.VPError):
        vp.vp_window_workspace_size(_shape(), w, 2)
    assert vp.vp_window_workspace_size(_shape(), _window(window=64), False) == 0  # a short walk needs none


# ---------------------------------------------------------------------------
# the reference's own pins
# ---------------------------------------------------------------------------
def test_reference_visibility():
    see = CO.visible(8, 2, 3, 2)
    # query 0 at position 6: sinks 0, 1 and 4 5 6; query 1 at 7: 5 6 7
    assert [np.nonzero(s)[0].tolist() for s in see] == [[0, 1, 4, 5, 6], [0, 1, 5, 6, 7]]
    assert CO.visible(1, 3, 0, 4).tolist() == [[False], [False], [True]]


def test_reference_attention_is_a_softmax():
    g = np.random.default_rng(0)
    q, K, V = g.standard_normal((1, 2, 4)), g.standard_normal((1, 6, 4)), g.standard_normal((1, 6, 4))
    r = CO.window_attention(q, K, V, 0, 0)
    e = np.exp(K[0] @ q[0, 1] / 2)
    np.testing.assert_allclose(r.out[0, 1], e @ V[0] / e.sum(), rtol=1e-12)
    np.testing.assert_allclose(r.weight.sum(), 2.0, rtol=1e-12)  # two heads' weights of one each


def test_reference_eviction():
    assert CO.kept_rows([5, 1, 9, 9, 2, 0], 6, 4, 1, 1).tolist() == [0, 2, 3, 5]
    assert CO.kept_rows([0, 7, 7, 7, 0], 5, 3, 0, 1).tolist() == [1, 2, 4]
    assert CO.kept_rows([0, math.nan, 7, math.inf, 0], 5, 2, 0, 0).tolist() == [1, 3]
    assert CO.kept_rows([3, 2], 2, 4, 1, 1).tolist() == [0, 1]
    assert CO.compact_segments([(0, 2), (2, 2), (4, 2)], [0, 2, 3, 5]) == [(0, 1), (1, 2), (3, 1)]


def test_sums_are_not_made_in_a_capture(monkeypatch):
    """A graph that made the sums would clear them in every replay."""
    import torch

    from _parity import small_workload
    from paper_2605_31457_amd import step
    ds = step.DeviceStep(small_workload(5, 1, 4, 1, 64, [50], [[]]), device="cpu")
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="before capturing"):
        ds.window_decode_attn(0, 4, sums=True)
    assert ds.attn_sum is None
