"""vp_window_decode_attn against the fp64 reference: windows, sinks, lengths from
none on, every type, head layout and cache layout, masked rows that hold anything,
running sums, graphs and streams."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from paper_2605_31457_amd import vp
from _cache import DEV, Caches, assert_attention, assert_sums, attention, i32, rounded, torch_dtype

pytestmark = pytest.mark.gpu


def draw(seed, B, T, Hq, Hkv, d, cap, dtype, scale=0.5):
    g = np.random.default_rng(seed)
    q = rounded(g.standard_normal((B, T, Hq, d)), dtype)
    K = rounded(scale * g.standard_normal((B, Hkv, cap, d)), dtype)
    V = rounded(scale * g.standard_normal((B, Hkv, cap, d)), dtype)
    return q, K, V


def on_device(q, dtype):
    return torch.from_numpy(q).to(torch_dtype(dtype)).to(DEV)


def check(q, K, V, lens, window, n_sink, dtype, order="bhs", page=0, sums=True, scale=0.0, ctx=""):
    """Both forms of the call (with and without sums) on one batch."""
    B, T, Hq, d = q.shape
    Hkv, cap = K.shape[1], K.shape[2]
    c = Caches(K, V, dtype, order, page, fill=float("nan"))
    qd = on_device(q, dtype)
    before = np.abs(np.random.default_rng(5).standard_normal((B, Hkv, cap))).astype(np.float32)
    for b, L in enumerate(lens):
        before[b, :, max(0, L - T):] = np.nan  # new rows and rows past the end hold anything
    runs = [None, torch.from_numpy(before).to(DEV)] if sums else [None]
    for s in runs:
        out = attention(c, qd, lens, window, n_sink, s, scale)
        for b, L in enumerate(lens):
            r = CO.window_attention(q[b], K[b, :, :L], V[b, :, :L], window, n_sink, scale if scale > 0 else None)
            name = f"{ctx} seq {b} L={L} window={window} sinks={n_sink} sums={s is not None}"
            assert_attention(out[b], r, dtype, L, name)
            if s is not None:
                assert_sums(s[b].cpu().numpy(), before[b], r, L, T, L, d, T * Hq // Hkv, name)


# lengths around the tile of 32 rows, the window and the sinks, in one batch
LENS = [0, 1, 2, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 200]


@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (1, 4), (31, 0), (32, 1), (33, 33), (64, 4), (100, 37),
                                           (40, 64), (500, 3), (2 ** 31 - 1, 2 ** 31 - 1), (7, 2 ** 31 - 1)])
@pytest.mark.parametrize("dtype,T,Hq,Hkv,d", [("bf16", 1, 14, 2, 128), ("f32", 2, 4, 1, 64)])
def test_windows_and_sinks(dtype, T, Hq, Hkv, d, window, n_sink):
    q, K, V = draw(window % 1000 + n_sink % 100, len(LENS), T, Hq, Hkv, d, 203, dtype)
    check(q, K, V, LENS, window, n_sink, dtype)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (0, 9), (520, 0), (576, 4), (600, 40), (640, 100), (550, 500),
                                           (900, 2 ** 31 - 1)])
@pytest.mark.parametrize("dtype,T,Hq,Hkv,d,page", [("bf16", 1, 4, 2, 128, 0), ("bf16", 3, 5, 1, 64, 16), ("f32", 2, 2, 2, 64, 0)])
def test_long_walks(dtype, T, Hq, Hkv, d, page, window, n_sink):
    """Walks of more tiles than one work-group takes, shared out by the lengths: ragged
    ones, empty sequences first, last and in between; the rows that nobody sees are NaN."""
    lens = [0, 1000, 1, 33, 0, 0, 519, 520, 521, 577, 640, 777, 992, 0]
    q, K, V = draw(window + n_sink % 97, len(lens), T, Hq, Hkv, d, 1001, dtype)
    for b, L in enumerate(lens):
        if window:
            K[b, :, min(n_sink, L):max(min(n_sink, L), L - T - window + 1)] = np.nan
            V[b, :, min(n_sink, L):max(min(n_sink, L), L - T - window + 1)] = np.nan
    check(q, K, V, lens, window, n_sink, dtype, page=page)


@pytest.mark.parametrize("B,Hkv,cap,window", [(65, 2, 700, 0), (130, 1, 700, 600), (300, 1, 620, 0), (500, 2, 560, 0)])
def test_long_walks_of_many_sequences(B, Hkv, cap, window):
    """More sequences than a wave has lanes."""
    q, K, V = draw(B, B, 1, 2 * Hkv, Hkv, 64, cap, "bf16")
    g = np.random.default_rng(B)
    lens = np.where(g.random(B) < 0.2, 0, g.integers(1, cap + 1, B)).tolist()
    check(q, K, V, lens, window, 0, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 1, 1), (1, 16, 1), (2, 6, 3), (3, 10, 2), (16, 2, 2), (4, 8, 2), (1, 5, 5)])
def test_heads_and_queries(dtype, d, T, Hq, Hkv):
    lens = [3, 50, 96, 161]  # (16 queries: the first sequence is shorter than they are)
    q, K, V = draw(T * 31 + Hq, len(lens), T, Hq, Hkv, d, 161, dtype)
    check(q, K, V, lens, 45, 5, dtype)
    check(q, K, V, lens, 0, 0, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order,page", [("bsh", 0), ("pad", 0), ("bhs", 1), ("bhs", 16), ("bsh", 32), ("pad", 64),
                                        ("bhs", 256)])
def test_cache_layouts(dtype, order, page):
    lens = [1, 40, 130, 259]
    q, K, V = draw(page + 3, len(lens), 2, 8, 2, 128, 260, dtype)
    for window, n_sink in ((0, 0), (70, 14), (33, 0)):
        check(q, K, V, lens, window, n_sink, dtype, order, page)


@pytest.mark.parametrize("dtype,B,T,Hq,Hkv,d,cap,window,n_sink,page", [
    ("bf16", 1, 1, 28, 4, 128, 3358, 1024, 4, 0),
    ("bf16", 1, 1, 28, 4, 128, 9000, 0, 0, 0),
    ("bf16", 3, 2, 64, 8, 128, 2500, 2000, 64, 16),
    ("bf16", 40, 1, 32, 8, 64, 700, 300, 4, 128),
    ("f32", 2, 1, 28, 4, 128, 1500, 0, 0, 0),
    ("f32", 70, 1, 16, 4, 64, 300, 100, 2, 32),
])
def test_larger_batches(dtype, B, T, Hq, Hkv, d, cap, window, n_sink, page):
    """One and several parts per KV head, more pairs than a round of work-groups."""
    q, K, V = draw(cap, B, T, Hq, Hkv, d, cap, dtype)
    lens = np.random.default_rng(cap).integers(1, cap + 1, B).tolist()
    lens[-1] = cap
    check(q, K, V, lens, window, n_sink, dtype, page=page)


@pytest.mark.parametrize("dtype,B,Hkv,d", [("bf16", 50, 8, 64), ("bf16", 66, 8, 64), ("bf16", 25, 8, 128),
                                           ("f32", 23, 8, 64), ("f32", 25, 8, 64)])
def test_windows_of_many_pairs(dtype, B, Hkv, d):
    """Batches on both sides of the numbers of pairs from which a work-group takes a whole
    window (of 20 tiles)."""
    q, K, V = draw(B, B, 1, Hkv, Hkv, d, 680, dtype)
    lens = np.random.default_rng(B).integers(0, 681, B).tolist()
    check(q, K, V, lens, 600, 4, dtype)


def test_more_pairs_than_work_groups():
    """600 (sequence, KV head) pairs: one part each, finished in one launch."""
    q, K, V = draw(1, 150, 1, 8, 4, 64, 90, "bf16")
    lens = np.random.default_rng(2).integers(0, 91, 150).tolist()
    check(q, K, V, lens, 50, 3, "bf16")


def test_no_workspace_where_none_is_needed():
    q, K, V = draw(2, 2, 1, 4, 2, 64, 200, "bf16")
    c, qd = Caches(K, V, "bf16"), on_device(q, "bf16")
    shape, w = c.shape(4), vp.vp_window(window=100, n_sink=4, sm_scale=0.0)
    assert vp.vp_window_workspace_size(shape, w) == 0
    out = torch.zeros_like(qd)
    seq_len = i32([200, 90])
    vp.vp_window_decode_attn(shape, c.layout(seq_len), w, qd, c.K, c.V, None, out, None, 0)
    assert torch.equal(out, attention(c, qd, [200, 90], 100, 4))


def test_tensors_elsewhere_are_refused():
    q, K, V = draw(2, 1, 1, 4, 2, 64, 50, "bf16")
    c, qd = Caches(K, V, "bf16"), on_device(q, "bf16")
    shape, w, seq_len = c.shape(4), vp.vp_window(window=0, n_sink=0, sm_scale=0.0), i32([50])
    out = torch.zeros_like(qd)
    for args in ((qd.cpu(), c.K, c.V, None, out), (qd, c.K, c.V.cpu(), None, out), (qd, c.K, c.V, torch.zeros(1, 2, 50), out)):
        with pytest.raises(ValueError):
            vp.vp_window_decode_attn(shape, c.layout(seq_len), w, *args, None, 1 << 30)
    assert float(out.abs().max()) == 0
    p = vp.vp_evict_params(budget=10, n_sink=0, n_recent=0)
    s = torch.ones(1, 2, 50, device=DEV)
    with pytest.raises(ValueError):
        vp.vp_evict(shape, c.layout(seq_len), p, s, c.K, c.V, torch.zeros(1, 10, dtype=torch.int32), s, None, seq_len,
                    torch.zeros(4096, dtype=torch.uint8, device=DEV))
    assert seq_len.tolist() == [50]


def test_logit_scale():
    q, K, V = draw(9, 2, 1, 8, 2, 128, 150, "bf16")
    check(q, K, V, [150, 77], 60, 2, "bf16", scale=0.37)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("T", [1, 3])
def test_masked_rows_hold_anything(dtype, d, bad, T):
    """Rows between the sinks and the window, past the end, and after a query's own
    position: NaN and infinities there reach no query that does not see them."""
    lens, window, n_sink = [170, 75, 40], 61, 5
    q, K, V = draw(4, 3, T, 10, 2, d, 180, dtype)
    Kb, Vb = K.copy(), V.copy()
    for b, L in enumerate(lens):
        lo = max(n_sink, L - T - window + 1)
        Kb[b, :, n_sink:lo] = Vb[b, :, n_sink:lo] = bad
        Kb[b, :, L:] = Vb[b, :, L:] = bad
    check(q, Kb, Vb, lens, window, n_sink, dtype)
    if T == 1:
        return
    # the last query's own row, and the oldest row of the first query's window: bad in
    # V (and K), seen by some queries only
    for at in (lambda L: L - 1, lambda L: max(n_sink, L - T - window + 1)):
        Kc, Vc = Kb.copy(), Vb.copy()
        for b, L in enumerate(lens):
            Kc[b, :, at(L)] = Vc[b, :, at(L)] = bad
        c = Caches(Kc, Vc, dtype)
        out = attention(c, on_device(q, dtype), lens, window, n_sink)
        for b, L in enumerate(lens):
            r = CO.window_attention(q[b], K[b, :, :L], V[b, :, :L], window, n_sink)
            for t in range(T):
                if r.seen[t, at(L)]:
                    continue
                one = CO.WindowResult(r.out[t:t + 1], r.weight, r.spread[t:t + 1], r.span, r.seen)
                assert_attention(out[b, t:t + 1], one, dtype, L, f"query {t} of {b}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_seen_rows_that_are_not_finite(dtype):
    """A NaN logit makes the head NaN in every part of the walk; an infinite value
    stays infinite; logits of -inf weigh nothing, and nothing but -inf gives zeros."""
    L, d = 900, 128
    q, K, V = draw(6, 1, 1, 4, 2, d, L, dtype)
    q[:] = np.abs(q) + 0.25
    q = rounded(q, dtype)
    Kn = K.copy()
    Kn[0, 0, 700] = np.nan
    out = attention(Caches(Kn, V, dtype), on_device(q, dtype), [L], 0, 0)[0, 0]
    assert bool(out[:2].isnan().all())
    r = CO.window_attention(q[0], K[0], V[0], 0, 0)
    one = CO.WindowResult(r.out[:, 2:], r.weight, r.spread[:, 2:], r.span, r.seen)
    assert_attention(out[None, 2:], one, dtype, L)
    Vi = V.copy()
    Vi[0, 1, 5, 3], Vi[0, 1, 800, 7] = np.inf, -np.inf
    out = attention(Caches(K, Vi, dtype), on_device(q, dtype), [L], 0, 0)[0, 0].double().cpu().numpy()
    assert np.all(out[2:, 3] == np.inf) and np.all(out[2:, 7] == -np.inf)
    assert np.all(np.isfinite(np.delete(out, [3, 7], 1)))
    Kz = K.copy()
    Kz[0, 0, 1::2] = -np.inf  # (q > 0: logits of -inf)
    Kz[0, 1] = -np.inf
    s = torch.ones(1, 2, L, device=DEV)
    out = attention(Caches(Kz, V, dtype), on_device(q, dtype), [L], 0, 0, s)[0]
    rz = CO.window_attention(q[0], Kz[0], V[0], 0, 0)
    assert_attention(out, rz, dtype, L)
    assert bool((out[0, 2:] == 0).all())
    assert bool((s[0, 0, 1:L - 1:2] == 1).all()) and bool((s[0, 1, :L - 1] == 1).all()) and float(s[0, 1, L - 1]) == 0


@pytest.mark.parametrize("dtype,page", [("bf16", 0), ("bf16", 64), ("f32", 0)])
def test_large_logits(dtype, page):
    """Logits of a few hundred, growing along the walk: the running maximum is raised
    again and again (the weights' error bound grows with the logits)."""
    q, K, V = draw(8, 2, 1, 8, 2, 64, 400, dtype, scale=1.0)
    K *= np.linspace(0.1, 24.0, 400)[None, None, :, None]
    K = rounded(K, dtype)
    check(q, K, V, [400, 333], 0, 0, dtype, page=page)
    check(q, K, V, [400, 333], 90, 2, dtype, page=page)


@pytest.mark.parametrize("dtype,page", [("bf16", 0), ("f32", 0), ("f32", 16)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("power", [9, 12, 20, 30])
def test_logits_whose_rounding_exceeds_the_softmax(dtype, page, sign, power):
    """Logits of up to 10^power, exact in fp32, the largest an eighth of that above the
    others: its row weighs 1 to the last bit and the others nothing, in walks of one part
    and of many."""
    for L in (300, 3001):
        q = np.zeros((1, 1, 4, 64))
        q[..., 0] = 1.0
        g = np.random.default_rng(power)
        K = np.zeros((1, 2, L, 64))
        K[0, :, :, 0] = sign * 10.0 ** power * g.uniform(0.25, 0.75, (2, L))
        best = g.integers(0, L, 2)
        for h in range(2):
            K[0, h, best[h], 0] = sign * 10.0 ** power * (0.875 if sign > 0 else 0.125)
        K = rounded(K, dtype)
        V = rounded(g.standard_normal((1, 2, L, 64)), dtype)
        s = torch.ones(1, 2, L, device=DEV)
        for sums in (None, s):
            out = attention(Caches(K, V, dtype, page=page), on_device(q, dtype), [L], 0, 0, sums, 1.0)
            out = out[0, 0].double().cpu().numpy()
            for h in range(4):
                assert np.array_equal(out[h], V[0, h // 2, best[h // 2]]), (L, h)
        want = np.ones((2, L))
        want[:, L - 1] = 0.0  # (the query's own row is new)
        want[[0, 1], best] += 2.0
        assert np.array_equal(s[0].double().cpu().numpy(), want)


def test_same_bits_every_time():
    q, K, V = draw(3, 4, 2, 28, 4, 128, 2100, "bf16")
    c = Caches(K, V, "bf16")
    lens = [2100, 1999, 64, 777]
    first = None
    for _ in range(4):
        s = torch.zeros(4, 4, 2100, device=DEV)
        out = attention(c, on_device(q, "bf16"), lens, 0, 0, s)
        first = first or (out, s)
        assert torch.equal(out, first[0]) and torch.equal(s, first[1])


def test_offsets_past_32_bits():
    """Sequences 6 GB apart: byte and element offsets of the second one pass 2^32."""
    d, Hkv, stride = 128, 2, (3 << 30)
    K, V = (torch.empty(stride + Hkv * 100 * d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    g = np.random.default_rng(1)
    q = rounded(g.standard_normal((2, 1, 4, d)), "bf16")
    k = rounded(0.5 * g.standard_normal((2, 2, Hkv, 100, d)), "bf16")
    views = []
    for x, src in ((K, k[0]), (V, k[1])):
        v = torch.as_strided(x, (2, Hkv, 100, d), (stride, 100 * d, d, 1))
        v.copy_(torch.from_numpy(src).to(torch.bfloat16))
        views.append(v)
    c = Caches.__new__(Caches)
    c.dtype, c.page, c.cap, c.table, (c.K, c.V) = "bf16", 0, 100, None, views
    for window, n_sink in ((0, 0), (50, 3)):
        out = attention(c, on_device(q, "bf16"), [99, 100], window, n_sink)
        for b, L in enumerate((99, 100)):
            r = CO.window_attention(q[b], k[0, b, :, :L], k[1, b, :, :L], window, n_sink)
            assert_attention(out[b], r, "bf16", L, f"seq {b}")


def test_lengths_past_the_capacity_are_clipped():
    q, K, V = draw(2, 2, 1, 4, 2, 64, 70, "bf16")
    c = Caches(K, V, "bf16")
    qd = on_device(q, "bf16")
    assert torch.equal(attention(c, qd, [1000, -5], 0, 0), attention(c, qd, [70, 0], 0, 0))


@pytest.mark.parametrize("sums", [False, True])
def test_captured_and_replayed(sums):
    """A captured call on a side stream: every replay gives the eager result."""
    q, K, V = draw(7, 4, 1, 28, 4, 128, 1500, "bf16")
    c = Caches(K, V, "bf16", page=32)
    qd, lens = on_device(q, "bf16"), i32([1500, 900, 31, 1])
    shape, w = c.shape(28), vp.vp_window(window=0 if sums else 700, n_sink=4, sm_scale=0.0)
    layout = c.layout(lens)
    nbytes = vp.vp_window_workspace_size(shape, w, sums)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(qd)
    s = torch.zeros(4, 4, 1500, device=DEV) if sums else None
    call = lambda: vp.vp_window_decode_attn(shape, layout, w, qd, c.K, c.V, s, out, ws, nbytes)
    call()
    torch.cuda.synchronize()
    want, want_s = out.clone(), s.clone() if sums else None
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for rep in range(4):
        out.fill_(3)
        if sums:
            s.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), rep
        if sums:
            assert torch.equal(s, want_s), rep


def test_two_streams_at_once():
    """Calls on two streams with a workspace each do not disturb one another."""
    q, K, V = draw(5, 2, 1, 28, 4, 128, 4000, "bf16")
    c = Caches(K, V, "bf16")
    qd, lens = on_device(q, "bf16"), i32([4000, 3500])
    shape, w = c.shape(28), vp.vp_window(window=0, n_sink=0, sm_scale=0.0)
    nbytes = vp.vp_window_workspace_size(shape, w, True)
    streams = [torch.cuda.Stream() for _ in range(2)]
    state = [(torch.empty(nbytes, dtype=torch.uint8, device=DEV), torch.zeros_like(qd),
              torch.zeros(2, 4, 4000, device=DEV)) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, (ws, out, s) in zip(streams, state):
            vp.vp_window_decode_attn(shape, c.layout(lens), w, qd, c.K, c.V, s, out, ws, nbytes, st)
    torch.cuda.synchronize()
    assert torch.equal(state[0][1], state[1][1]) and torch.equal(state[0][2], state[1][2])
    r = CO.window_attention(q[0], K[0], V[0], 0, 0)
    assert_attention(state[0][1][0], r, "bf16", 4000)
