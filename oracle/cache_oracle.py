"""fp64 reference of the bounded-cache calls (vp_window_decode_attn, vp_evict).

TEST INFRASTRUCTURE, like vp_oracle: the definitions written out in float64,
one sequence at a time, without code shared with the library.

* Query t of T is the token at position p_t = L - T + t and sees the positions
  j <= p_t with j < n_sink or j > p_t - window (window 0: every j <= p_t).
* A query that sees nothing, or whose logits are all -inf, gives zeros.
* Eviction keeps the first n_sink, the last n_recent and the best-scored rows
  in between, ties to the lower position; a NaN score is the largest.
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import numpy as np

__all__ = ["WindowResult", "visible", "window_attention", "kept_rows", "compact_segments"]


@dataclass
class WindowResult:
    out: np.ndarray      # [T, Hq, d]
    weight: np.ndarray   # [Hkv, L] attention weight of every row, all queries and heads of the group
    spread: np.ndarray   # [T, Hq, d] sum_j A_j |V_j|
    span: np.ndarray     # [T, Hq] largest sum_i |q_i K_ji| * scale over the visible rows
    seen: np.ndarray     # [T, L] visibility


def visible(L: int, T: int, window: int, n_sink: int) -> np.ndarray:
    see = np.zeros((T, L), bool)
    for t in range(T):
        p = L - T + t
        for j in range(min(p, L - 1) + 1):
            see[t, j] = window == 0 or j < n_sink or j > p - window
    return see


def window_attention(q, K, V, window: int, n_sink: int, sm_scale: float | None = None) -> WindowResult:
    """q [T, Hq, d], K and V [Hkv, L, d] (any float type)."""
    q, K, V = (np.asarray(x, np.float64) for x in (q, K, V))
    T, Hq, d = q.shape
    Hkv, L, _ = K.shape
    G = Hq // Hkv
    scale = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    seen = visible(L, T, window, n_sink)
    r = WindowResult(np.zeros((T, Hq, d)), np.zeros((Hkv, L)), np.zeros((T, Hq, d)), np.zeros((T, Hq)), seen)
    for t in range(T):
        rows = np.nonzero(seen[t])[0]
        if rows.size == 0:
            continue
        for h in range(Hq):
            g = h // G
            with np.errstate(invalid="ignore"):
                z = scale * (K[g, rows] @ q[t, h])
            m = np.max(z)
            if m == -np.inf:
                continue
            e = np.exp(z - m)
            A = e / e.sum()
            live = A != 0.0  # a row of logit -inf is absent
            r.out[t, h] = A[live] @ V[g, rows[live]]
            r.spread[t, h] = A[live] @ np.abs(V[g, rows[live]])
            r.span[t, h] = abs(scale) * np.max(np.abs(K[g, rows[live]]) @ np.abs(q[t, h]))
            r.weight[g, rows] += A
    return r


def kept_rows(score, L: int, budget: int, n_sink: int, n_recent: int) -> np.ndarray:
    """Positions that stay, ascending; score [>= L] of the rows."""
    if L <= budget:
        return np.arange(L)
    rank = lambda j: (0, 0.0, j) if math.isnan(score[j]) else (1, -float(score[j]), j)
    mid = sorted(range(n_sink, L - n_recent), key=rank)[:budget - n_sink - n_recent]
    return np.array(list(range(n_sink)) + sorted(mid) + list(range(L - n_recent, L)), np.int64)


def compact_segments(segments, kept) -> list[tuple[int, int]]:
    """The segments {start, length} in the numbering of the kept rows."""
    kept = np.asarray(kept)
    return [(int((kept < s).sum()), int(((kept >= s) & (kept < s + n)).sum())) for s, n in segments]
