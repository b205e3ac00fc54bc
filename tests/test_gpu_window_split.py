"""Batches of many (sequence, KV head) pairs on both sides of the rules by which a work-group
takes a whole walk: one full sequence among short ones, full ones, windows that cut the walks
and windows that do not."""
import numpy as np
import pytest

from test_gpu_window import check, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,T,B,Hkv,d,whole,dealt", [("bf16", 1, 165, 2, 64, 69, 72), ("bf16", 2, 40, 8, 64, 51, 54),
                                                         ("f32", 1, 40, 8, 64, 51, 54), ("bf16", 1, 40, 8, 128, 51, 54)])
@pytest.mark.parametrize("window", [0, 2 ** 31 - 1, 1200, 700])
def test_one_full_sequence_among_short_ones(dtype, T, B, Hkv, d, whole, dealt, window):
    """Capacities on both sides of the one from which walks without a window (or with one that
    cuts little) are dealt; 700 cuts them to half, and is taken whole either way."""
    for tiles in (whole, dealt):
        cap = 32 * tiles - 5
        q, K, V = draw(B + tiles, B, T, Hkv, Hkv, d, cap, dtype)
        lens = np.random.default_rng(B).integers(0, 70, B).tolist()
        lens[B // 2] = cap
        check(q, K, V, lens, window, 4, dtype)


@pytest.mark.parametrize("tiles", [32, 35])
def test_lengths_of_every_size(tiles):
    cap = 32 * tiles
    q, K, V = draw(tiles, 50, 1, 8, 4, 64, cap, "bf16")
    check(q, K, V, np.linspace(0, cap, 50).astype(int).tolist(), 0, 0, "bf16")
