"""The range of the sums of attention over 16-, 32- and 4-bit caches: values up to the stated limit."""
import numpy as np
import pytest
import torch

from _cache import DEV, Caches, attention, i32, torch_dtype
from _kv4 import Four
from paper_2605_31457_amd import vp

pytestmark = pytest.mark.gpu


def _attention4(c, q, L, dtype, scale):
    shape, w = c.shape(q.shape[2], dtype), vp.vp_window(window=0, n_sink=0, sm_scale=scale)
    seq_len, out = i32([L]), torch.full_like(q, 7.0)
    n = vp.vp_kv4_workspace_size(shape, w)
    ws = torch.full((max(n, 1),), 0xff, dtype=torch.uint8, device=DEV)
    vp.vp_kv4_decode_attn(shape, c.layout(seq_len), w, q, c.struct(), out, ws, n)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L", [896, 4096])
def test_largest_values(L, d, four, dtype):
    """Values of 2^111 / L (L up to a power of two) where weights are as large as they get before the running maximum is
    raised: it is by products that exceed it by 8 / (scale log2 e) = 33, but next to 2^29, where numbers are 64
    apart, 2^29 + 33 is 2^29 + 64, so the second half's products, 64 above the first's, raise nothing and weigh
    2^(64 8 / 33) = 2^15.5.

    All values are the same, so the output is that value, off by the orders of its sum and the
    normaliser's: of positive terms, at most 3 L / 4 + 200 additions in a wave and the joins (three parts of every weight), each
    off by a whole step of float32 at most; both sums, and the output's rounding."""
    value = 2.0 ** 111 / 2.0 ** np.ceil(np.log2(L))
    K = np.zeros((1, L, d))
    K[:, :, 0] = 2.0 ** 14
    K[:, L // 2:, 32] = 64.0
    V = np.full((1, L, d), value)
    q = np.zeros((1, 1, 2, d))
    q[..., 0], q[..., 32] = 2.0 ** 15, 1.0
    qd = torch.from_numpy(q).to(torch_dtype(dtype)).to(DEV)
    scale = 8 / 33 / 1.4426950408889634
    if four:
        c = Four(1, 1, L, d)
        c.put([K], [V])
        got = _attention4(c, qd, L, dtype, scale)
    else:
        got = attention(Caches(K[None], V[None], dtype), qd, [L], 0, 0, scale=scale)
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got))
    bound = 2 * (3 * L / 4 + 200) * 2.0 ** -23 + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
    assert np.all(np.abs(got / value - 1) <= bound), np.max(np.abs(got / value - 1)) / bound
