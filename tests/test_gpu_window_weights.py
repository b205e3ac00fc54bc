"""The bits of the softmax weights that reach the outputs of vp_window_decode_attn in bf16."""
import numpy as np
import pytest
import torch

from _cache import DEV, EPS, Caches, attention, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("live", [4, 5, 6])
@pytest.mark.parametrize("L,window,n_sink", [(33, 0, 0), (200, 150, 4), (2000, 0, 0), (2000, 1500, 4)])
@pytest.mark.parametrize("d,page", [(128, 0), (64, 16)])
def test_outputs_of_values_that_cancel(live, L, window, n_sink, d, page):
    """`live` rows share the weight, all others have a logit 1000 below (weight 2^-1443, 0).
    The values nearly cancel, so an output's own rounding hides nothing of the weights' error.

    Error in steps of EPS, relative to sum_j A_j |V_j|: the products and the scale are exact; the
    exponent is at most 1.4 with a constant and a product rounded (2 EPS of it, times ln 2: 2),
    2^x is off by a step (2), so 4, and the joins of waves and of parts twice as much again
    (none for walks of one part; 12 in all). Every weight enters as 3 products that are exact,
    each added with one step's error at most (2), and in each of the two joins once more: 6 per
    live row, and 4. Then half a step of bf16. (The normaliser's error is relative to the output.)"""
    g = np.random.default_rng(live + L)
    H, scale = 8, 0.5
    at = np.sort(g.choice(np.arange(L - 30, L), live, replace=False))
    k = g.integers(0, 32, (H, live)) / 16.0
    w = np.exp(scale * (k - k.max(1, keepdims=True)))
    v = rounded(g.standard_normal((H, live, d)), "bf16")
    for r in (live - 2, live - 1):  # the last two take away what the others add up to
        v[:, r] = 0.0
        v[:, r] = rounded(-np.einsum("hl,hld->hd", w, v) / w[:, r, None], "bf16")
    K = np.zeros((1, H, L, d))
    K[..., 0] = -2000.0
    K[0, :, at, 0] = k.T
    V = rounded(g.standard_normal((1, H, L, d)), "bf16")
    V[0, :, at] = v.transpose(1, 0, 2)
    q = np.zeros((1, 1, H, d))
    q[..., 0] = 1.0
    assert np.array_equal(K, rounded(K, "bf16"))
    A = w / w.sum(1, keepdims=True)
    want, spread = np.einsum("hl,hld->hd", A, v), np.einsum("hl,hld->hd", A, np.abs(v))
    bound = (12 + 10 * live if L == 2000 else 4 + 6 * live) * EPS * spread
    bound = bound + 2.0 ** -8 * (np.abs(want) + bound) + 1e-37
    qd = torch.from_numpy(q).to(torch.bfloat16).to(DEV)
    for sums in (None, torch.zeros(1, H, L, device=DEV)):
        out = attention(Caches(K, V, "bf16", page=page), qd, [L], window, n_sink, sums, scale)
        worst = np.max(np.abs(out[0, 0].double().cpu().numpy() - want) / bound)
        assert worst <= 1.0, worst
