"""4-bit caches: appending, reading back and attention, against the reference."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from oracle import kv4_oracle as KO
from paper_2605_31457_amd import vp
from _cache import DEV, Caches, i32, rounded
from _kv4 import Four, New, assert_rounded, attention_bound, cos_sin, rope

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# rows in and out
# ---------------------------------------------------------------------------
def _held(x):
    """The values that a 4-bit row holds of x."""
    return KO.decode(*KO.quantise(x))


def _same(a, b):
    return np.array_equal(a, b, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,rot,sections,interleaved", [
    (28, 4, 128, 128, None, False), (4, 1, 64, 64, None, False), (16, 16, 64, 32, None, True),
    (6, 3, 128, 16, None, False), (8, 2, 128, 128, (16, 24, 24), False), (8, 2, 64, 64, (8, 12, 12), True),
    (8, 2, 128, 0, None, False)])
@pytest.mark.parametrize("page", [0, 16, 64])
def test_append_rows(dtype, Hq, Hkv, d, rot, sections, interleaved, page):
    """Codes and scales of the new rows are exactly those of the 64-bit values; nothing else is written."""
    rng = np.random.default_rng(page + rot)
    lens, counts = [70, 5, 0, 33], [37, 5, 0, 2]
    c = Four(4, Hkv, 80, d, page=page, gap=16)
    new = New(rng, 44, Hq, Hkv, d, dtype)
    n_axes = len(sections) if sections else 1
    pos = rng.integers(0, 90, (n_axes, 44))
    table = cos_sin(90, max(rot, 2), 1)
    t, p = torch.from_numpy(table).to(DEV), i32(pos.tolist())
    q_out = torch.full((44, Hq, d), 7.0, dtype=new.dev.dtype, device=DEV)
    before = [x.clone() for x in c.codes + c.scales]
    seq_len, off = i32(lens), i32([0, 37, 42, 42, 44])
    vp.vp_append_kv4(c.shape(Hq, dtype), c.layout(seq_len), rope(t, p, sections, interleaved) if rot else None,
                     new.struct(off), q_out, c.struct())
    torch.cuda.synchronize()
    kr = KO.rotate(new.k, table, pos, rot, sections, interleaved)
    assert_rounded(q_out.double().cpu().numpy(), KO.rotate(new.q, table, pos, rot, sections, interleaved), dtype, "q")
    K, V = c.get(80)
    i = 0
    for b, (L, n) in enumerate(zip(lens, counts)):
        for got, want in ((K[b], kr), (V[b], new.v)):
            assert _same(got[:, L - n:L], _held(want[i:i + n].transpose(1, 0, 2))), (b, "rows")
        i += n
    # everything else: put the old rows back and nothing differs
    for x, old in zip(c.codes + c.scales, before):
        for b, (L, n) in enumerate(zip(lens, counts)):
            for j in range(L - n, L):
                at = (int(c.table[b, j // page]), j % page) if page else (b, j)
                x[at[0], :, at[1]] = old[at[0], :, at[1]]
        assert bool((x == old).all())


def test_borders():
    """Values on and next to the borders of codes and scales, zeros, the smallest and largest
    numbers, infinities and NaN."""
    d = 128
    blocks = []
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, 7.0])
    for e in (-130, -126, -125, -124, -20, 0, 3, 100, 123, 125):
        s = 2.0 ** e
        near = np.concatenate([mids, np.nextafter(mids.astype(np.float32), np.float32(9)).astype(float),
                               np.nextafter(mids.astype(np.float32), np.float32(0)).astype(float)])
        for top in (4.0, 6.0, 7.0, float(np.nextafter(np.float32(7), np.float32(9))), 8.0):
            x = near[near <= top][:31]
            x = np.concatenate([x * np.where(np.arange(x.size) % 2, -1, 1), np.zeros(31 - x.size), [top]])
            blocks.append(x * s)
    big = float(np.finfo(np.float32).max)
    blocks += [np.zeros(32), -np.zeros(32), np.full(32, 2.0 ** -149), np.full(32, big), np.linspace(-big, big, 32)]
    for bad in (np.inf, -np.inf, np.nan):
        x = np.ones(32)
        x[7] = bad
        blocks.append(x)
    while len(blocks) % 4:
        blocks.append(np.ones(32))
    with np.errstate(over="ignore"):
        x = np.stack(blocks).reshape(-1, 1, d).astype(np.float32).astype(float)
    n = x.shape[0]
    new = New.__new__(New)
    new.set(np.concatenate([x, x, -x], 1), 1, 1, "f32")
    c = Four(1, 1, n, d)
    seq_len, off = i32([n]), i32([0, n])
    q_out = torch.zeros(n, 1, d, device=DEV)
    vp.vp_append_kv4(c.shape(1, "f32"), c.layout(seq_len), None, new.struct(off), q_out, c.struct())
    K, V = c.get(n)
    assert _same(q_out.double().cpu().numpy(), x)
    assert _same(K[0], _held(x.transpose(1, 0, 2))) and _same(V[0], _held(-x.transpose(1, 0, 2)))
    # and back: zeros, normal numbers, NaN
    for dtype in ("f32", "bf16"):
        o = Caches(np.zeros((1, 1, n, d)), np.zeros((1, 1, n, d)), dtype)
        vp.vp_kv4_read(o.shape(1), o.layout(seq_len), c.struct(), None, o.K, o.V)
        Kr, Vr = o.get()
        assert _same(Kr, K) and _same(Vr, V)


def test_border_of_the_64_bit_value():
    """Rotated elements that round to a code's border in 32 bits and lie beside it in 64."""
    d, n = 64, 64
    rng = np.random.default_rng(5)
    x = np.zeros((n, 3, d))
    x[:, :, 0:32] = 1.0
    x[:, :, 32:] = 2.0 ** -30 * np.where(rng.random((n, 1, 32)) < 0.5, -1, 1)
    x[:, :, 31] = 4.0  # the block's largest: scale 1
    table = np.ones((1, 64), np.float32)
    table[:, :31] = np.resize([0.25, 0.75, 1.25, 1.75, 2.5, 3.5], 31)
    x = rounded(x, "f32")
    new = New.__new__(New)
    new.set(x, 1, 1, "f32")
    c = Four(1, 1, n, d)
    t = torch.from_numpy(table).to(DEV)
    seq_len, off = i32([n]), i32([0, n])
    vp.vp_append_kv4(c.shape(1, "f32"), c.layout(seq_len), rope(t), new.struct(off),
                     torch.zeros(n, 1, d, device=DEV), c.struct())
    kr = KO.rotate(x[:, 1:2], table, np.zeros((1, n), int), 64)
    assert len(np.unique(_held(kr)[:, 0, 0])) == 2  # (the borders fall either way)
    assert _same(c.get(n)[0][0], _held(kr.transpose(1, 0, 2)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,page,order", [(128, 0, "bhs"), (64, 0, "bsh"), (128, 16, "bhs"), (64, 128, "pad")])
@pytest.mark.parametrize("some", [False, True])
def test_read(dtype, d, page, order, some):
    """Rows from `first` on come back exactly; other rows keep their bits."""
    rng = np.random.default_rng(d + page)
    lens = [1, 300, 0, 64, 77, 500]
    B, Hkv, cap = 6, 3, 290
    K0, V0 = (rounded(rng.standard_normal((B, Hkv, cap, d)), dtype) for _ in range(2))
    o = Caches(K0, V0, dtype, order=order, page=page, seed=3)
    c = Four(B, Hkv, cap, d, page=page, table=o.table)
    rows = [rng.standard_normal((Hkv, cap, d)) * 2.0 ** rng.integers(-9, 9, (Hkv, cap, 1)) for _ in range(2 * B)]
    c.put(rows[:B], rows[B:])
    first = [0, 13, 5, 64, -3, 289] if some else [0] * B
    seq_len = i32(lens)
    f = i32(first) if some else None
    vp.vp_kv4_read(o.shape(Hkv), o.layout(seq_len), c.struct(), f, o.K, o.V)
    torch.cuda.synchronize()
    for got, old, src in zip(o.get(), (K0, V0), (rows[:B], rows[B:])):
        for b in range(B):
            L, lo = min(lens[b], cap), max(0, first[b])
            lo = min(lo, L)
            assert np.array_equal(got[b][:, lo:L], _held(src[b])[:, lo:L]), b
            assert np.array_equal(got[b][:, :lo], old[b][:, :lo]) and np.array_equal(got[b][:, L:], old[b][:, L:]), b


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def _attention(c, q, lens, window, n_sink, dtype, scale=0.0, stream=None):
    """One vp_kv4_decode_attn call; q: device [B, T, Hq, d]."""
    B, T, Hq, d = q.shape
    shape, w = c.shape(Hq, dtype, T), vp.vp_window(window=window, n_sink=n_sink, sm_scale=scale)
    seq_len = i32(lens)
    out = torch.full_like(q, 7.0)
    nbytes = vp.vp_kv4_workspace_size(shape, w)
    ws = torch.full((nbytes + 64,), 0xff, dtype=torch.uint8, device=DEV)
    vp.vp_kv4_decode_attn(shape, c.layout(seq_len), w, q, c.struct(), out, ws, nbytes, stream)
    torch.cuda.synchronize()
    assert bool((ws[nbytes:] == 0xff).all())
    return out


def _case(rng, lens, Hq, Hkv, d, dtype, T, cap=None, page=0, spread=1.0, gap=0):
    B = len(lens)
    cap = cap or max(max(lens), 1)
    K = [rng.standard_normal((Hkv, min(max(L, 0), cap), d)) * 2.0 ** rng.integers(-3, 3, (Hkv, 1, d // 32)).repeat(32, -1) for L in lens]
    V = [rng.standard_normal((Hkv, min(max(L, 0), cap), d)) * spread for L in lens]
    c = Four(B, Hkv, cap, d, page=page, seed=1, gap=gap)
    c.put(K, V)
    q = rounded(rng.standard_normal((B, T, Hq, d)), dtype)
    qd = torch.from_numpy(q).to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)
    return c, qd, q, [_held(x) for x in K], [_held(x) for x in V]


def _check(got, q, K, V, window, n_sink, dtype, scale=None, ctx=""):
    got = got.double().cpu().numpy()
    for b in range(len(K)):
        n = K[b].shape[1]
        r = CO.window_attention(q[b], K[b], V[b], window, n_sink, scale)
        bound = attention_bound(r, dtype, n, q.shape[-1], q.shape[1] * q.shape[2])
        assert np.all(np.isfinite(got[b])), (ctx, b)
        worst = np.max(np.abs(got[b] - r.out) / bound)
        assert worst <= 1.0, f"{ctx} sequence {b}: {worst:.2f} times the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,T", [(28, 4, 128, 1), (14, 2, 128, 2), (4, 1, 64, 1), (3, 3, 64, 4), (16, 1, 128, 1), (2, 2, 64, 16)])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (40, 5), (7, 0), (33, 70)])
def test_short(dtype, Hq, Hkv, d, T, window, n_sink):
    """Walks of one work-group: lengths from none and one to a few tiles."""
    rng = np.random.default_rng(Hq + T)
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 64, 95, 200]
    c, qd, q, K, V = _case(rng, lens, Hq, Hkv, d, dtype, T)
    _check(_attention(c, qd, lens, window, n_sink, dtype), q, K, V, window, n_sink, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,T,page", [(28, 4, 128, 1, 0), (14, 2, 128, 2, 16), (8, 2, 64, 1, 32), (8, 2, 64, 3, 128)])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (700, 33), (1, 1)])
def test_long(dtype, Hq, Hkv, d, T, page, window, n_sink):
    """Walks dealt to several work-groups and joined; room past the longest sequence."""
    rng = np.random.default_rng(Hq + page)
    lens = [1701, 3, 1024, 0, 640]
    c, qd, q, K, V = _case(rng, lens, Hq, Hkv, d, dtype, T, cap=2500, page=page, gap=16)
    _check(_attention(c, qd, lens, window, n_sink, dtype), q, K, V, window, n_sink, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 32])
def test_masked_rows_have_no_influence(dtype, page):
    """NaN in the rows that a query does not see: before the window, after its position, past
    the end, and in the whole blocks beside."""
    rng = np.random.default_rng(3)
    Hq, Hkv, d, T, W, S = 8, 2, 128, 3, 50, 5
    lens = [150, 49, 6]
    c, qd, q, K, V = _case(rng, lens, Hq, Hkv, d, dtype, T, cap=192, page=page)
    ref = _attention(c, qd, lens, W, S, dtype)
    for x in c.scales:  # every row that no query sees, and one that only the last two see
        for b, L in enumerate(lens):
            for j in range(192):
                if j >= L or (j >= S and j <= L - T - W):
                    at = (int(c.table[b, j // page]), j % page) if page else (b, j)
                    x[at[0], :, at[1]] = 255
    assert bool((_attention(c, qd, lens, W, S, dtype) == ref).all())
    # the last query's own row is seen by it alone
    for x in c.scales:
        for b, L in enumerate(lens):
            at = (int(c.table[b, (L - 1) // page]), (L - 1) % page) if page else (b, L - 1)
            x[at[0], :, at[1]] = 255
    got = _attention(c, qd, lens, W, S, dtype)
    assert bool((got[:, :T - 1] == ref[:, :T - 1]).all()) and bool(got[:, T - 1].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits_and_values(dtype):
    """Logits of thousands, values that cancel, scales from 2^-60 to 2^60."""
    rng = np.random.default_rng(4)
    Hq, Hkv, d, lens = 4, 2, 64, [300]
    c, qd, q, K, V = _case(rng, lens, Hq, Hkv, d, dtype, 1, spread=2.0 ** 60)
    _check(_attention(c, qd, lens, 0, 0, dtype, scale=0.5), q, K, V, 0, 0, dtype, 0.5)
    c, qd, q, K, V = _case(rng, lens, Hq, Hkv, d, dtype, 1, spread=2.0 ** -60)
    _check(_attention(c, qd, lens, 0, 0, dtype, scale=40.0), q, K, V, 0, 0, dtype, 40.0)


def test_infinite_queries():
    """Infinite logits of one sign: rows of -inf alone give zeros, as in the 16-bit call."""
    Hkv, d, L = 1, 64, 40
    K = np.ones((Hkv, L, d))
    V = np.ones((Hkv, L, d))
    c = Four(1, Hkv, L, d)
    c.put([K], [V])
    for dtype in ("bf16", "f32"):
        q = torch.full((1, 1, 2, d), -float("inf"), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device=DEV)
        q[0, 0, 1] = 1.0
        got = _attention(c, q, [L], 0, 0, dtype)
        assert bool((got[0, 0, 0] == 0).all()) and bool((got[0, 0, 1] == 1).all()), dtype


@pytest.mark.parametrize("B,Hkv,cap,window", [(100, 1, 3000, 0), (70, 2, 2500, 1900), (300, 1, 700, 0), (260, 3, 300, 64)])
def test_many_sequences(B, Hkv, cap, window):
    """More sequences than a wave has lanes, dealt and whole."""
    rng = np.random.default_rng(B)
    lens = np.where(rng.random(B) < 0.1, cap, rng.integers(0, 40, B)).tolist()
    c, qd, q, K, V = _case(rng, lens, 3 * Hkv, Hkv, 64, "bf16", 1, cap=cap, page=32)
    _check(_attention(c, qd, lens, window, 3, "bf16"), q, K, V, window, 3, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_heads(dtype):
    rng = np.random.default_rng(12)
    lens = [70, 33]
    c, qd, q, K, V = _case(rng, lens, 512, 256, 64, dtype, 1)
    _check(_attention(c, qd, lens, 0, 0, dtype), q, K, V, 0, 0, dtype)


def test_heads_outside_sequences():
    """Planes of a head before those of a sequence ([Hkv][B][rows]), and lengths outside the capacity."""
    rng = np.random.default_rng(13)
    B, Hkv, cap, d = 3, 2, 48, 128
    c, qd, q, K, V = _case(rng, [48, 20, 0], 8, Hkv, d, "bf16", 1, cap=cap)
    want = _attention(c, qd, [48, 20, 0], 0, 0, "bf16")
    c.codes = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in c.codes]
    c.scales = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in c.scales]
    assert bool((_attention(c, qd, [60, 20, -5], 0, 0, "bf16") == want).all())
    new = New(rng, 4, 8, Hkv, d, "bf16", queries=False)
    seq_len, off = i32([48, 20, 9]), i32([0, 2, 2, 4])
    vp.vp_append_kv4(c.shape(8, "bf16"), c.layout(seq_len), None, new.struct(off), None, c.struct())
    Kg, Vg = c.get(cap)
    for b, (lo, hi, i) in {0: (46, 48, 0), 2: (7, 9, 2)}.items():
        assert np.array_equal(Kg[b][:, lo:hi], _held(new.k[i:i + 2].transpose(1, 0, 2)))
        assert np.array_equal(Vg[b][:, lo:hi], _held(new.v[i:i + 2].transpose(1, 0, 2)))
    assert np.array_equal(Kg[1][:, :20], K[1]) and np.array_equal(Kg[0][:, :46], K[0][:, :46])


def test_far_offsets():
    """Planes beyond 2^32 bytes: a block far into a pool, and a sequence far into a batch."""
    rng = np.random.default_rng(9)
    Hq, Hkv, d, page, L = 4, 1, 128, 1 << 16, 333
    n = 1200  # blocks of 4 MiB: 4.7 GiB of codes
    c = Four.__new__(Four)
    c.page, c.cap, c.d = page, page, d
    c.table = i32([[n - 1]])
    c.codes = [torch.zeros(n, Hkv, page, d // 2, dtype=torch.uint8, device=DEV) for _ in range(2)]
    c.scales = [torch.full((n, Hkv, page, d // 32), 127, dtype=torch.uint8, device=DEV) for _ in range(2)]
    new = New(rng, L, Hq, Hkv, d, "bf16")
    seq_len, off = i32([L]), i32([0, L])
    q_out = torch.zeros(L, Hq, d, dtype=torch.bfloat16, device=DEV)
    vp.vp_append_kv4(c.shape(Hq, "bf16"), c.layout(seq_len), None, new.struct(off), q_out, c.struct())
    K, V = _held(new.k.transpose(1, 0, 2)), _held(new.v.transpose(1, 0, 2))
    got = _attention(c, q_out[-1:].view(1, 1, Hq, d), [L], 0, 0, "bf16")
    _check(got, new.q[-1:].reshape(1, 1, Hq, d), [K], [V], 0, 0, "bf16")
    assert not bool(c.codes[0][:n - 1].any())
    del c
    torch.cuda.empty_cache()


def test_same_bits_again_and_other_streams():
    rng = np.random.default_rng(10)
    lens = [2100, 900, 1500]
    c, qd, q, K, V = _case(rng, lens, 28, 4, 128, "bf16", 1, cap=2500, page=32)
    ref = _attention(c, qd, lens, 0, 0, "bf16")
    s = torch.cuda.Stream()
    for stream in (None, s, s, None):
        assert bool((_attention(c, qd, lens, 0, 0, "bf16", stream=stream) == ref).all())
