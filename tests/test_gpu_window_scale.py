"""vp_window_decode_attn at the ends of the logit scale's range."""
import numpy as np
import pytest
import torch

from _cache import DEV, Caches, attention, rounded, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1e30, 2.3e38, 2.4e38, float(np.finfo(np.float32).max)])
@pytest.mark.parametrize("dtype,L", [("bf16", 60), ("bf16", 2000), ("f32", 60), ("f32", 2000)])
def test_the_largest_scales(dtype, L, scale):
    """Products in steps of 1: the row of the largest weighs 1, the others nothing."""
    q = np.zeros((1, 1, 4, 64))
    q[..., 0] = 1.0
    g = np.random.default_rng(L)
    K = np.zeros((1, 2, L, 64))
    K[0, :, :, 0] = g.integers(-40, 40, (2, L))
    best = g.integers(0, L - 1, 2)
    K[0, [0, 1], best, 0] = 41.0
    V = rounded(g.standard_normal((1, 2, L, 64)), dtype)
    s = torch.ones(1, 2, L, device=DEV)
    for sums in (None, s):
        out = attention(Caches(K, V, dtype), torch.from_numpy(q).to(torch_dtype(dtype)).to(DEV), [L], 0, 0, sums, scale)
        for h in range(4):
            assert np.array_equal(out[0, 0, h].double().cpu().numpy(), V[0, h // 2, best[h // 2]])
    want = np.ones((2, L))
    want[:, L - 1] = 0.0  # (the query's own row is new)
    want[[0, 1], best] += 2.0
    assert np.array_equal(s[0].double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_smallest_scale(dtype):
    """Logits of next to nothing: every row weighs the same."""
    L = 64
    g = np.random.default_rng(1)
    q, K = rounded(g.standard_normal((1, 1, 4, 64)), dtype), rounded(g.standard_normal((1, 2, L, 64)), dtype)
    s = torch.zeros(1, 2, L, device=DEV)
    attention(Caches(K, np.ones_like(K), dtype), torch.from_numpy(q).to(torch_dtype(dtype)).to(DEV), [L], 0, 0, s, 1e-37)
    # (products below 100 and a scale of 1e-37: weights of 1 / 64 to the last bit, two heads' each)
    assert bool((s == 2.0 / 64).all())
