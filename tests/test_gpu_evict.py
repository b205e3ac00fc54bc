"""vp_evict against the definition: kept rows exactly, the compacted caches, sums and
segments bit for bit, and everything behind them untouched."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from paper_2605_31457_amd import vp
from _cache import DEV, Caches, i32, rounded

pytestmark = pytest.mark.gpu


def evict(c, Hq, sums, lens, budget, n_sink, n_recent, groups, segs=None, in_place=True, T=1, stream=None):
    """One call. Returns (kept [B, U, C], sums_out, new_len, segments) as numpy; the
    caches change in place. in_place: sums, lengths and segments do too."""
    B, Hkv, cap = sums.shape
    shape = c.shape(Hq, T, vp.VP_SCOPE_KV_GROUP if groups else vp.VP_SCOPE_SEQUENCE, cap)
    p = vp.vp_evict_params(budget=budget, n_sink=n_sink, n_recent=n_recent)
    seq_len = i32(lens)
    off = seg = seg_out = None
    if segs is not None:
        off = i32(np.cumsum([0] + [len(s) for s in segs]).tolist())
        seg = i32([x for s in segs for x in s] or [(0, 0)])
        seg_out = seg if in_place else torch.full_like(seg, -3)
    sums = sums.clone()
    sums_out = sums if in_place else torch.full_like(sums, -2.0)
    new_len = seq_len if in_place else torch.full_like(seq_len, -1)
    U = Hkv if groups else 1
    kept = torch.full((B * U, budget), -9, dtype=torch.int32, device=DEV)
    nbytes = vp.vp_evict_workspace_size(shape, p)
    ws = torch.full((nbytes + 64,), 0xff, dtype=torch.uint8, device=DEV)
    vp.vp_evict(shape, c.layout(seq_len, off, seg), p, sums, c.K, c.V, kept, sums_out, seg_out, new_len, ws, nbytes,
                stream)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0xff).all())
    return (kept.view(B, U, budget).cpu().numpy(), sums_out.cpu().numpy(), new_len.cpu().numpy(),
            None if seg_out is None else seg_out.cpu().numpy())


def check(K, V, sums, lens, budget, n_sink, n_recent, groups, dtype="bf16", order="bhs", page=0, segs=None, Hq=None):
    B, Hkv, cap, d = K.shape
    Hq = Hq or Hkv
    dev_sums = torch.from_numpy(sums).to(DEV)
    for in_place in (True, False):
        c = Caches(K, V, dtype, order, page, fill=5.0)
        spare = None
        if page:
            spare = sorted(set(range(c.K.shape[0])) - set(c.table.flatten().tolist()))
        kept, new_sums, new_len, new_segs = evict(c, Hq, dev_sums, lens, budget, n_sink, n_recent, groups, segs, in_place)
        K2, V2 = c.get()
        if page:
            assert bool((c.K[spare] == 5).all()) and bool((c.V[spare] == 5).all())
        i = 0
        for b, L in enumerate(lens):
            n = min(L, budget)
            assert new_len[b] == n
            for u in range(Hkv if groups else 1):
                score = sums[b, u] if groups else sums[b].astype(np.float64).sum(0).astype(np.float32)
                want = CO.kept_rows(score, L, budget, n_sink, n_recent)
                ctx = f"seq {b} L={L} list {u} in_place={in_place}"
                assert np.array_equal(kept[b, u, :n], want), ctx
                assert np.all(kept[b, u, n:] == -1), ctx
                for g in [u] if groups else range(Hkv):
                    for got, src in ((K2, K), (V2, V)):
                        assert np.array_equal(got[b, g, :n], src[b, g, want], equal_nan=True), f"{ctx} head {g}"
                        assert np.array_equal(got[b, g, n:], src[b, g, n:], equal_nan=True), f"{ctx} head {g}: behind"
                    assert np.array_equal(new_sums[b, g, :n], sums[b, g, want], equal_nan=True), f"{ctx} sums of {g}"
                    behind = sums[b, g, n:] if in_place else np.full(cap - n, -2.0, np.float32)
                    assert np.array_equal(new_sums[b, g, n:], behind, equal_nan=True), f"{ctx} sums behind"
            if segs is not None:
                for s in CO.compact_segments(segs[b], want):
                    assert tuple(new_segs[i]) == s, f"seq {b} segment {i}"
                    i += 1


def draw(seed, B, Hkv, cap, d=64, dtype="bf16"):
    g = np.random.default_rng(seed)
    K, V = (rounded(g.standard_normal((B, Hkv, cap, d)), dtype) for _ in range(2))
    sums = np.exp(2 * g.standard_normal((B, Hkv, cap))).astype(np.float32)
    return K, V, sums


LENS = [0, 1, 63, 64, 65, 66, 100, 200, 301]


@pytest.mark.parametrize("groups", [False, True])
@pytest.mark.parametrize("n_sink,n_recent", [(0, 0), (4, 0), (0, 64), (64, 0), (30, 34), (3, 17)])
def test_budgets_and_protected_rows(groups, n_sink, n_recent):
    K, V, sums = draw(n_sink + n_recent, len(LENS), 3, 303)
    check(K, V, sums, LENS, 64, n_sink, n_recent, groups)


@pytest.mark.parametrize("budget", [1, 2, 31, 299, 300, 301, 302, 5000])
def test_any_budget(budget):
    K, V, sums = draw(budget, 2, 2, 301)
    check(K, V, sums, [301, 150], budget, min(1, budget - 1), 0, True)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("order,page", [("bhs", 0), ("bsh", 0), ("pad", 0), ("bhs", 1), ("bsh", 16), ("pad", 32),
                                        ("bhs", 128)])
def test_cache_layouts(dtype, d, order, page):
    K, V, sums = draw(page + d, 3, 2, 700, d, dtype)
    check(K, V, sums, [700, 420, 333], 350, 4, 50, page % 2 == 0, dtype, order, page)


@pytest.mark.parametrize("cap,budget", [(2000, 1000), (4000, 100), (8000, 7000), (16000, 8000), (32768, 20000),
                                        (32769, 16384), (70000, 35000)])
@pytest.mark.parametrize("groups", [False, True])
def test_key_counts(cap, budget, groups):
    """Rows whose keys fit 2 to 32 registers a thread, and longer ones."""
    K, V, sums = draw(cap, 1, 2, cap)
    check(K, V, sums, [cap - 1], budget, 14, 50, groups)


@pytest.mark.parametrize("groups", [False, True])
def test_ties_go_to_the_lower_position(groups):
    K, V, sums = draw(1, 3, 2, 500)
    sums[0] = 1.0
    sums[1] = np.random.default_rng(0).integers(0, 4, (2, 500)).astype(np.float32)
    sums[2] = 0.0
    sums[2, :, ::3] = -0.0
    check(K, V, sums, [500, 480, 490], 200, 2, 20, groups)


def test_sums_that_are_not_finite():
    K, V, sums = draw(2, 2, 2, 400)
    sums[:, :, 10:60] = np.nan
    sums[:, :, 100:150] = np.inf
    sums[:, :, 200:300] = -np.inf
    sums[1] = np.nan
    check(K, V, sums, [400, 400], 130, 1, 5, True)


def test_scores_are_added_in_64_bits():
    """Small sums beside a large one: added in 32 bits, in any order, they would be lost
    and the tie would go to the lower position."""
    K, V, sums = draw(3, 1, 4, 300)
    sums[:] = np.float32(2.0 ** 24)
    sums[0, 1:, 1::2] += np.float32(1.0) * 2  # 2^24 + 2: representable
    sums[0, 0] = 1.0
    check(K, V, sums, [300], 120, 0, 10, False)


def test_rows_that_hold_anything_move_as_they_are():
    K, V, sums = draw(4, 1, 2, 200)
    K[0, :, 50:100] = np.nan
    V[0, :, 20:70] = np.inf
    V[0, :, 120:] = -np.inf
    check(K, V, sums, [190], 90, 2, 9, True)


def test_segments_follow_their_rows():
    """Segments cut, emptied and shifted, none, and 256 of them; in the layout's own array."""
    K, V, sums = draw(5, 5, 2, 1200)
    sums[0, :, 30:200] = 0.0  # the first image goes whole
    segs = [[(30, 170), (300, 400)], [], [(0, 1)], [(2 * i, 1) for i in range(256)], [(10, 50), (1100, 90)]]
    check(K, V, sums, [1200, 1000, 900, 1111, 600], 500, 5, 100, False, segs=segs)


def test_segments_outside_the_sequence_are_clipped():
    K, V, sums = draw(6, 1, 1, 300)
    c = Caches(K, V, "bf16")
    # reaching past the length, overlapping its predecessor, of negative length
    kept, _, _, seg = evict(c, 1, torch.from_numpy(sums).to(DEV), [250], 100, 0, 0, False,
                            [[(20, 100), (60, 100), (200, 500), (230, -4)]], in_place=False)
    rows = kept[0, 0]
    count = lambda a, z: int(((rows >= a) & (rows < z)).sum())
    assert seg.tolist() == [[count(0, 20), count(20, 120)], [count(0, 120), count(120, 160)],
                            [count(0, 200), count(200, 250)], [count(0, 250), 0]]


def test_lengths_outside_the_capacity_are_clipped():
    K, V, sums = draw(8, 2, 2, 150)
    dev = torch.from_numpy(sums).to(DEV)
    runs = []
    for lens in ([900, -7], [150, 0]):
        c = Caches(K, V, "bf16")
        runs.append(evict(c, 2, dev, lens, 64, 2, 9, True) + tuple(c.get()))
    for x, y in zip(*runs):
        assert x is None and y is None or np.array_equal(x, y)
    assert runs[0][2].tolist() == [64, 0]


@pytest.mark.parametrize("dtype,d,Hkv,groups", [("bf16", 128, 4, True), ("f32", 128, 2, False), ("bf16", 64, 8, False)])
def test_many_sequences(dtype, d, Hkv, groups):
    K, V, sums = draw(11, 24, Hkv, 900, d, dtype)
    lens = np.random.default_rng(3).integers(1, 901, 24).tolist()
    check(K, V, sums, lens, 400, 4, 64, groups, dtype, page=32)


def test_offsets_past_32_bits():
    """Sequences 6 GB apart: byte and element offsets of the second one pass 2^32."""
    d, Hkv, cap, stride = 128, 2, 300, 3 << 30
    K, V, sums = draw(21, 2, Hkv, cap, d)
    c = Caches.__new__(Caches)
    c.dtype, c.page, c.cap, c.table = "bf16", 0, cap, None
    views = []
    for src in (K, V):
        x = torch.empty(stride + Hkv * cap * d, dtype=torch.bfloat16, device=DEV)
        views.append(torch.as_strided(x, (2, Hkv, cap, d), (stride, cap * d, d, 1)))
        views[-1].copy_(torch.from_numpy(src).to(torch.bfloat16))
    c.K, c.V = views
    kept, _, new_len, _ = evict(c, 4, torch.from_numpy(sums).to(DEV), [300, 299], 150, 4, 20, True)
    got = c.get()
    for b, L in enumerate((300, 299)):
        for h in range(Hkv):
            rows = CO.kept_rows(sums[b, h], L, 150, 4, 20)
            assert np.array_equal(kept[b, h], rows)
            for x, src in zip(got, (K, V)):
                assert np.array_equal(x[b, h, :150], src[b, h, rows]) and np.array_equal(x[b, h, 150:], src[b, h, 150:])


def test_evicting_again_and_again():
    """In place, round after round with new rows appended, as a decode loop does."""
    K, V, sums = draw(12, 2, 2, 400)
    c = Caches(K, V, "bf16")
    want_K, want_V, want_s, lens = K.copy(), V.copy(), sums.copy(), [400, 310]
    g = np.random.default_rng(9)
    for step in range(6):
        dev = torch.from_numpy(want_s).to(DEV)
        kept, new_s, new_len, _ = evict(c, 2, dev, lens, 256, 3, 40, True)
        for b in range(2):
            for h in range(2):
                rows = CO.kept_rows(want_s[b, h], lens[b], 256, 3, 40)
                assert np.array_equal(kept[b, h, :len(rows)], rows), step
                for x in (want_K, want_V, want_s):
                    x[b, h, :len(rows)] = x[b, h, rows]
        assert np.array_equal(new_s, want_s)
        got = c.get()
        assert np.array_equal(got[0], want_K) and np.array_equal(got[1], want_V), step
        lens = [int(n) + 50 + 30 * b for b, n in enumerate(new_len)]
        for b in range(2):
            new = slice(int(new_len[b]), lens[b])
            want_s[b, :, new] = np.exp(g.standard_normal((2, lens[b] - int(new_len[b]))))


@pytest.mark.parametrize("groups", [False, True])
def test_captured_and_replayed(groups):
    K, V, sums = draw(13, 3, 4, 5000, 128)
    c = Caches(K, V, "bf16", page=64)
    shape = c.shape(28, 1, int(groups), 5000)
    p = vp.vp_evict_params(budget=2500, n_sink=4, n_recent=200)
    s, lens = torch.from_numpy(sums).to(DEV), i32([5000, 4000, 2000])
    kept = torch.zeros(12 if groups else 3, 2500, dtype=torch.int32, device=DEV)
    s_out, new_len = torch.zeros_like(s), torch.zeros_like(lens)
    ws = torch.empty(vp.vp_evict_workspace_size(shape, p), dtype=torch.uint8, device=DEV)
    layout = c.layout(lens)
    K0, V0 = c.K.clone(), c.V.clone()
    call = lambda: vp.vp_evict(shape, layout, p, s, c.K, c.V, kept, s_out, None, new_len, ws)
    call()
    torch.cuda.synchronize()
    want = [x.clone() for x in (c.K, c.V, kept, s_out, new_len)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for rep in range(4):
        c.K.copy_(K0)
        c.V.copy_(V0)
        for x in (kept, s_out, new_len):
            x.fill_(-1)
        s_out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((c.K, c.V, kept, s_out, new_len), want):
            assert torch.equal(x, y), rep


def test_two_streams_at_once():
    K, V, sums = draw(14, 2, 4, 6000, 128)
    a, b = Caches(K, V, "bf16"), Caches(K, V, "bf16")
    shape = a.shape(28, 1, 1, 6000)
    p = vp.vp_evict_params(budget=3000, n_sink=4, n_recent=200)
    s, lens = torch.from_numpy(sums).to(DEV), i32([6000, 5000])
    runs = []
    for c in (a, b):
        runs.append((c, torch.cuda.Stream(), torch.zeros(8, 3000, dtype=torch.int32, device=DEV), torch.zeros_like(s),
                     torch.zeros_like(lens),
                     torch.empty(vp.vp_evict_workspace_size(shape, p), dtype=torch.uint8, device=DEV)))
    torch.cuda.synchronize()
    for _ in range(10):
        for c, st, kept, s_out, new_len, ws in runs:
            vp.vp_evict(shape, c.layout(lens), p, s, c.K, c.V, kept, s_out, None, new_len, ws, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(a.K, b.K) and torch.equal(a.V, b.V) and torch.equal(runs[0][2], runs[1][2])
