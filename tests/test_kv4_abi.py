"""Host side of appending and of 4-bit caches (no GPU): refusals before anything is enqueued,
struct sizes, workspace sizes, and the reference itself."""
import ctypes
import math

import numpy as np
import pytest

from oracle import kv4_oracle as KO
from paper_2605_31457_amd import vp

PTR = 1 << 20  # an aligned address that nothing dereferences


def _shape(**kw):
    s = dict(batch=2, n_q_heads=28, n_kv_heads=4, head_dim=128, dtype=vp.VP_BF16, max_seq_len=4096, max_vis=1296,
             max_segs=1, k_cap=64, block_size=0, n_queries=1, kv_stride_b=4 * 4096 * 128, kv_stride_h=4096 * 128,
             kv_stride_s=128)
    s.update(kw)
    return vp.vp_shape(**s)


def _layout(**kw):
    return vp.vp_layout(**dict(dict(seq_len=PTR, vis_seg_off=None, vis_seg=None, block_table=None), **kw))


def _rope(section=(0, 0, 0, 0), **kw):
    r = dict(cos_sin=PTR, n_pos=4096, rot_dim=128, interleaved=0, n_axes=1, pos=None)
    r.update(kw)
    return vp.vp_rope(section=(ctypes.c_int32 * 4)(*section), **r)


def _tokens(**kw):
    t = dict(q=PTR, k=PTR, v=PTR, q_stride=36 * 128, k_stride=36 * 128, v_stride=36 * 128, new_off=PTR, n_tokens=5)
    t.update(kw)
    return vp.vp_tokens(**t)


def _four(**kw):
    c = dict(k_codes=PTR, k_scales=PTR, v_codes=2 * PTR, v_scales=2 * PTR, code_stride_b=4 * 4096 * 64,
             code_stride_h=4096 * 64, scale_stride_b=4 * 4096 * 4, scale_stride_h=4096 * 4)
    c.update(kw)
    return vp.vp_kv4(**c)


def _refused(status, call, *args):
    with pytest.raises(vp.VPError) as e:
        call(*args)
    assert status in str(e.value)


def _append(shape=None, layout=None, rope=None, tokens=None, q_out=3 * PTR, K=PTR, V=2 * PTR):
    vp.vp_append_kv(shape or _shape(), layout or _layout(), rope, tokens or _tokens(), q_out, K, V, 0)


def _append4(shape=None, layout=None, rope=None, tokens=None, q_out=3 * PTR, cache=None):
    vp.vp_append_kv4(shape or _shape(), layout or _layout(), rope, tokens or _tokens(), q_out, cache or _four(), 0)


def _read(shape=None, layout=None, cache=None, first=None, K=PTR, V=2 * PTR):
    vp.vp_kv4_read(shape or _shape(), layout or _layout(), cache or _four(), first, K, V, 0)


def _attend(shape=None, layout=None, window=None, q=PTR, cache=None, out=PTR, ws=PTR, nbytes=1 << 40):
    vp.vp_kv4_decode_attn(shape or _shape(), layout or _layout(), window or vp.vp_window(window=0, n_sink=0, sm_scale=0.0),
                          q, cache or _four(), out, ws, nbytes, 0)


def test_struct_sizes():
    assert ctypes.sizeof(vp.vp_rope) == 48 and ctypes.sizeof(vp.vp_tokens) == 64 and ctypes.sizeof(vp.vp_kv4) == 64


@pytest.mark.parametrize("call", [_append, _append4])
@pytest.mark.parametrize("status,kw", [
    ("VP_ERR_NULL", dict(cos_sin=None)), ("VP_ERR_SHAPE", dict(cos_sin=PTR + 8)), ("VP_ERR_RANGE", dict(n_pos=0)),
    ("VP_ERR_SHAPE", dict(rot_dim=0)), ("VP_ERR_SHAPE", dict(rot_dim=24)), ("VP_ERR_SHAPE", dict(rot_dim=144)),
    ("VP_ERR_SHAPE", dict(rot_dim=-16)), ("VP_ERR_RANGE", dict(interleaved=2)), ("VP_ERR_RANGE", dict(n_axes=0)),
    ("VP_ERR_RANGE", dict(n_axes=5, pos=PTR)), ("VP_ERR_SHAPE", dict(pos=PTR + 2)),
    ("VP_ERR_NULL", dict(n_axes=3, section=(16, 24, 24, 0))),
    ("VP_ERR_SHAPE", dict(n_axes=3, pos=PTR, section=(16, 24, 20, 0))),
    ("VP_ERR_SHAPE", dict(n_axes=3, pos=PTR, section=(16, 24, 20, 4))),
    ("VP_ERR_SHAPE", dict(n_axes=2, pos=PTR, section=(30, 34, 0, 0))),
    ("VP_ERR_SHAPE", dict(n_axes=2, pos=PTR, section=(-4, 68, 0, 0))),
])
def test_rotation(call, status, kw):
    _refused(status, call, None, None, _rope(**kw))


@pytest.mark.parametrize("call", [_append, _append4])
@pytest.mark.parametrize("status,kw", [
    ("VP_ERR_NULL", dict(k=None)), ("VP_ERR_NULL", dict(v=None)), ("VP_ERR_NULL", dict(q=None)),
    ("VP_ERR_SHAPE", dict(q=PTR + 8)), ("VP_ERR_SHAPE", dict(k=PTR + 2)), ("VP_ERR_SHAPE", dict(v=PTR + 4)),
    ("VP_ERR_SHAPE", dict(q_stride=28 * 128 - 8)), ("VP_ERR_SHAPE", dict(k_stride=0)), ("VP_ERR_SHAPE", dict(v_stride=-512)),
    ("VP_ERR_SHAPE", dict(k_stride=515)), ("VP_ERR_SHAPE", dict(new_off=PTR + 1)), ("VP_ERR_RANGE", dict(n_tokens=-1)),
    ("VP_ERR_RANGE", dict(n_tokens=(1 << 24) + 1)), ("VP_ERR_SHAPE", dict(new_off=None, n_tokens=0)),
    ("VP_ERR_SHAPE", dict(new_off=None)),  # 5 tokens for 2 sequences of one query
])
def test_tokens(call, status, kw):
    _refused(status, call, None, None, None, _tokens(**kw))


@pytest.mark.parametrize("call", [_append, _append4])
def test_append_arguments(call):
    _refused("VP_ERR_NULL", call, None, _layout(seq_len=None))
    _refused("VP_ERR_NULL", call, _shape(block_size=32), None)
    _refused("VP_ERR_NULL", call, None, None, None, None, None)  # queries without q_out
    _refused("VP_ERR_SHAPE", call, None, None, None, None, PTR + 8)
    _refused("VP_ERR_SHAPE", call, None, None, None, None, PTR)  # q_out is q, a column of one product
    _refused("VP_ERR_DTYPE", call, _shape(dtype=4))
    _refused("VP_ERR_UNSUPPORTED", call, _shape(head_dim=96))


@pytest.mark.parametrize("call", [_append, _append4])
def test_no_tokens(call):
    """Nothing to append: nothing is enqueued, and empty tensors' addresses do not matter."""
    call(None, None, _rope(), _tokens(n_tokens=0, k=None, v=None, q=None), None)


def test_append_caches():
    _refused("VP_ERR_NULL", _append, None, None, None, None, 3 * PTR, None)
    _refused("VP_ERR_SHAPE", _append, None, None, None, None, 3 * PTR, PTR + 8)
    _refused("VP_ERR_SHAPE", _append, None, None, None, None, 3 * PTR, PTR, PTR)
    _refused("VP_ERR_SHAPE", _append, _shape(kv_stride_h=64), None, None, None, 3 * PTR)


@pytest.mark.parametrize("status,kw", [
    ("VP_ERR_NULL", dict(k_codes=None)), ("VP_ERR_NULL", dict(v_scales=None)), ("VP_ERR_SHAPE", dict(k_codes=PTR + 8)),
    ("VP_ERR_SHAPE", dict(v_scales=PTR + 4)), ("VP_ERR_SHAPE", dict(code_stride_b=-16)),
    ("VP_ERR_SHAPE", dict(code_stride_h=4096 * 64 + 8)), ("VP_ERR_SHAPE", dict(scale_stride_h=4096 * 4 + 4)),
])
def test_cache_of_4_bits(status, kw):
    _refused(status, _append4, None, None, None, None, 3 * PTR, _four(**kw))
    _refused(status, _read, None, None, _four(**kw))
    _refused(status, _attend, None, None, None, PTR, _four(**kw))


@pytest.mark.parametrize("kw", [dict(v_codes=PTR), dict(v_scales=PTR), dict(code_stride_h=4096 * 64 - 16),
                                dict(scale_stride_h=0), dict(code_stride_b=4096 * 64), dict(scale_stride_b=16)])
def test_rows_that_overlap(kw):
    _refused("VP_ERR_SHAPE", _append4, None, None, None, None, 3 * PTR, _four(**kw))


@pytest.mark.parametrize("page", [1, 2, 8])
def test_small_blocks(page):
    s, l = _shape(block_size=page), _layout(block_table=PTR)
    _refused("VP_ERR_UNSUPPORTED", _append4, s, l, None, None, 3 * PTR)
    _refused("VP_ERR_UNSUPPORTED", _read, s, l)
    _refused("VP_ERR_UNSUPPORTED", _attend, s, l)


def test_read_and_attention():
    _refused("VP_ERR_NULL", _read, None, None, None, None, None)
    _refused("VP_ERR_SHAPE", _read, None, None, None, None, PTR, PTR)
    _refused("VP_ERR_SHAPE", _read, None, None, None, PTR + 2)
    _refused("VP_ERR_SHAPE", _read, _shape(kv_stride_h=64))
    _refused("VP_ERR_NULL", _attend, None, None, None, None)
    _refused("VP_ERR_NULL", _attend, None, None, None, PTR, None, None)
    _refused("VP_ERR_SHAPE", _attend, None, None, None, PTR + 8)
    _refused("VP_ERR_RANGE", _attend, None, None, vp.vp_window(window=-1, n_sink=0, sm_scale=0.0))
    _refused("VP_ERR_RANGE", _attend, None, None, vp.vp_window(window=0, n_sink=0, sm_scale=math.nan))
    _refused("VP_ERR_WORKSPACE", _attend, None, None, None, PTR, None, PTR, None)
    _refused("VP_ERR_WORKSPACE", _attend, None, None, None, PTR, None, PTR, PTR, 100)


def test_workspace_sizes():
    w = vp.vp_window(window=0, n_sink=0, sm_scale=0.0)
    assert vp.vp_kv4_workspace_size(_shape(max_seq_len=64), w) == 0
    assert 0 < vp.vp_kv4_workspace_size(_shape(), w) < 64 << 20
    for B in (1, 7, 64, 4096, 65535):
        assert vp.vp_kv4_workspace_size(_shape(batch=B, max_seq_len=1 << 20), w) >= 0


# ---------------------------------------------------------------------------
# the reference
# ---------------------------------------------------------------------------
def test_reference_quantise():
    x = np.zeros(32)
    x[:10] = [0.25, 0.26, 0.75, -1.25, 1.75, 2.5, 3.5, -5.0, 5.1, 7.0]
    code, byte = KO.quantise(x)
    assert byte.tolist() == [127]
    assert KO.decode(code, byte)[:10].tolist() == [0.0, 0.5, 1.0, -1.0, 2.0, 2.0, 4.0, -4.0, 6.0, 6.0]
    x[9] = 7.0000005
    assert KO.quantise(x)[1].tolist() == [128]
    assert KO.quantise(np.full(32, 3.5))[1].tolist() == [126]
    assert KO.quantise(np.zeros(32))[1].tolist() == [2]
    x[3] = np.nan
    assert np.isnan(KO.decode(*KO.quantise(x))).all()


def test_reference_error():
    """An element is off by a step of 2 scales, halved, at most: the largest is 3.5 scales or more."""
    x = np.random.default_rng(0).standard_normal((500, 64))
    e = np.abs(KO.decode(*KO.quantise(x)) - x).reshape(500, 2, 32)
    assert np.all(e <= np.abs(x).reshape(500, 2, 32).max(-1, keepdims=True) / 7 * 2)
    exact = KO.decode(np.arange(32).astype(np.uint8) % 16, np.array([140], np.uint8))
    assert np.array_equal(KO.decode(*KO.quantise(exact)), exact)


def test_reference_rotate():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 64))
    a = rng.uniform(-3, 3, (5, 16))
    table = np.concatenate([np.cos(a), np.sin(a)], 1)
    pos = np.array([[4, 0, 2]])
    y = KO.rotate(x, table, pos, 32)
    z = (x[..., :16] + 1j * x[..., 16:32]) * np.exp(1j * a[pos[0]])[:, None]
    assert np.allclose(y[..., :16], z.real) and np.allclose(y[..., 16:32], z.imag) and np.array_equal(y[..., 32:], x[..., 32:])
    y = KO.rotate(x, table, pos, 32, interleaved=True)
    z = (x[..., 0:32:2] + 1j * x[..., 1:32:2]) * np.exp(1j * a[pos[0]])[:, None]
    assert np.allclose(y[..., 0:32:2], z.real) and np.allclose(y[..., 1:32:2], z.imag)
    two = KO.rotate(x, table, np.array([[0, 0, 0], [4, 0, 2]]), 32, (4, 12))
    assert np.allclose(two[..., :4], KO.rotate(x, table, [[0, 0, 0]], 32)[..., :4])
    assert np.allclose(two[..., 4:16], KO.rotate(x, table, pos, 32)[..., 4:16])
