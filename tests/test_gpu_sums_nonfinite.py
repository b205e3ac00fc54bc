"""The running sums of vp_window_decode_attn beside logits that are not finite."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from _cache import DEV, EPS, Caches, attention, rounded, torch_dtype, weight_error

pytestmark = pytest.mark.gpu


def draw(seed, B, T, Hq, Hkv, d, cap, dtype):
    g = np.random.default_rng(seed)
    q = rounded(g.standard_normal((B, T, Hq, d)), dtype)
    K = rounded(0.5 * g.standard_normal((B, Hkv, cap, d)), dtype)
    V = rounded(0.5 * g.standard_normal((B, Hkv, cap, d)), dtype)
    return q, K, V


@pytest.mark.parametrize("where", ["sink", "oldest", "middle", "last"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("T", [1, 2, 3])
@pytest.mark.parametrize("dtype,d,page,cap,lens,window,n_sink", [
    ("bf16", 128, 0, 130, [75, 44, 66, 130], 61, 5),      # one work-group per pair; rows 5 to 13 of 75 in nobody's view
    ("f32", 64, 16, 130, [75, 44, 66, 130], 61, 5),
    ("bf16", 64, 16, 1100, [620, 1100, 606, 33], 600, 5),  # walks that are shared out
    ("bf16", 128, 0, 1100, [650, 1100, 33, 645], 600, 40),
    ("f32", 128, 0, 1100, [650, 1100, 33, 645], 600, 40),
])
def test_sums_beside_logits_that_are_not_finite(dtype, d, page, cap, lens, window, n_sink, T, bad, where):
    """A NaN or +inf logit makes the weights of the queries that see its row NaN, on the
    rows that they see. Rows that no query sees keep their bits, those between the sinks and
    the window in a tile that is walked among them, and rows that only other queries see have
    their sums."""
    at = {"sink": lambda L: 2, "oldest": lambda L: max(n_sink, L - T - window + 1), "middle": lambda L: L - 20,
          "last": lambda L: L - 1}[where]
    q, K, V = draw(T + cap, len(lens), T, 4, 2, d, cap, dtype)
    Kb = K.copy()
    for b, L in enumerate(lens):
        Kb[b, 0, at(L), 3] = bad  # (of one KV head: the other's sums are all finite)
    c = Caches(Kb, V, dtype, page=page)
    before = np.random.default_rng(5).standard_normal((len(lens), 2, cap)).astype(np.float32)
    before[:, :, ::7] = -0.0
    s = torch.from_numpy(before).to(DEV)
    attention(c, torch.from_numpy(q).to(torch_dtype(dtype)).to(DEV), lens, window, n_sink, s)
    got = s.cpu().numpy()
    gaps = 0
    for b, L in enumerate(lens):
        with np.errstate(invalid="ignore"):
            r = CO.window_attention(q[b], Kb[b, :, :L], V[b, :, :L], window, n_sink)
        clean = CO.window_attention(q[b], K[b, :, :L], V[b, :, :L], window, n_sink)
        seen = np.zeros(cap, bool)
        seen[:L] = r.seen.any(0)
        gaps += int((~seen[:L]).sum())
        same = got[b].view(np.uint32) == before[b].view(np.uint32)
        assert np.all(same[:, ~seen]), f"seq {b}: rows that no query sees"
        want = before[b].astype(np.float64)
        want[:, L - T:L] = 0.0
        want[:, :L] += r.weight
        assert np.array_equal(np.isnan(got[b][:, seen]), np.isnan(want[:, seen])), f"seq {b}: NaN sums"
        # the finite ones: the bounds of finite inputs (the bad row aside, the logits are the clean ones')
        add = np.where(np.isfinite(want[:, :L]), r.weight, 0.0)
        bound = (weight_error(clean, d, L, 2 * T) + (2 * T + 1) * EPS) * add + EPS * np.abs(want[:, :L]) + 1e-37
        fine = np.isfinite(want[:, :L]) & seen[:L]
        assert np.all(np.abs(got[b][:, :L] - want[:, :L])[fine] <= bound[fine]), f"seq {b}: finite sums"
    assert gaps
