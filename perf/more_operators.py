"""Caches that grow and caches held in 4 bits, as measurable cases.

  op "append"   vp_append_kv: the queries and keys of new tokens are rotated by
                their positions, and keys and values go to the last rows of
                their sequences' caches;
  op "append4"  vp_append_kv4, the same into a 4-bit cache, and vp_kv4_read of
                the new rows: what the cache holds of them, as a chunk's own
                attention needs it;
  op "read4"    vp_kv4_read: rows of a 4-bit cache back in a cache of 16 or 32
                bits, on which the calls of the method run;
  op "attn4"    vp_kv4_decode_attn: attention of a step's queries over a 4-bit
                cache, all of it or a window and the first tokens.

A 4-bit row holds one sign, exponent and mantissa code (E2M1) per element and a
power of two (E8M0) per 32 elements, the least whose sevenfold is not below the
largest of them.

Lengths vary over the batch between `len_min` and `len_max`, new tokens between
`new_min` and `new_max`, and depend on the case alone (`mix`); `room` rows past the
longest sequence are free. Keys have a few wide channels, as rotated keys do;
where attention reads them, one row in fifty points along its KV group's
queries.
"""
import ctypes
import math
import random

import torch

own = False  # true: the framework's calls; false: the plain form

DEVICE = "cuda:0"
SPIKE_NATS = 4.0  # mean logit gain of an attended row

# name -> (query heads, KV heads, head_dim): the attention shapes of the
# repository's configurations and tests
HEADS = {
    "28/4": (28, 4, 128),
    "64/8": (64, 8, 128),
    "32/8": (32, 8, 128),
    "32/32": (32, 32, 128),
    "16/16x64": (16, 16, 64),
    "4/1x64": (4, 1, 64),
}

_BASE = dict(op="attn4", heads="28/4", dtype="bf16", batch=1, len_min=3358, len_max=3358, new_min=1, new_max=1, room=0,
             page=0, rot=128, axes=0, interleaved=False, fused=True, queries=1, window=0, sinks=4, mix=1)


def _case(name, **kw):
    c = dict(_BASE, name=name)
    for k, v in kw.items():
        assert k in c, k
        c[k] = v
    if "len_max" in kw and "len_min" not in kw:
        c["len_min"] = c["len_max"]
    if "new_max" in kw and "new_min" not in kw:
        c["new_min"] = c["new_max"]
    return c


def listed():
    return [
        # the smallest call: one token of a tiny draft model
        _case("app_tiny_f32", op="append", heads="4/1x64", dtype="f32", len_max=384, rot=64),
        # a serving batch's decode step, one token per sequence, paged in blocks of 32 rows
        _case("app_b64_step", op="append", batch=64, len_min=500, len_max=2477, page=32, mix=3),
        # prompts with images: ragged chunks, positions of three axes, 72B-class heads
        _case("app_prefill", op="append", heads="64/8", batch=8, len_min=1500, len_max=4096, new_min=800, new_max=2048,
              axes=3, mix=7),
        # into 4 bits: one user's decode step
        _case("app4_b1_step", op="append4", len_max=3358),
        # a serving batch's step, two drafted tokens per sequence, paged, half of every head rotated
        _case("app4_b64_step", op="append4", batch=64, len_min=500, len_max=2477, new_max=2, page=32, rot=64, mix=3),
        # prompts: ragged chunks of up to 2k tokens, three axes
        _case("app4_prefill", op="append4", batch=8, len_min=1500, len_max=4096, new_min=1000, new_max=2048, axes=3, mix=5),
        # one user's context back in 16 bits
        _case("read4_b1_3k", op="read4"),
        # a paged serving batch's contexts
        _case("read4_b16", op="read4", batch=16, len_min=5000, len_max=12288, page=32, mix=4),
        # attention: a short fp32 sequence, launches and dependent loads
        _case("attn4_tiny_f32", heads="4/1x64", dtype="f32", len_max=384),
        # one user's step over 8k tokens
        _case("attn4_b1_8k", len_max=8192),
        # a paged serving batch, two queries per sequence, windows of 4k, sequences
        # shorter than that among them; the system text stays visible
        _case("attn4_b16_paged_q2", batch=16, len_min=500, len_max=12288, window=4096, sinks=14, page=32, queries=2, mix=3),
        # the largest: 64 contexts of 32k tokens
        _case("attn4_b64_32k", batch=64, len_max=32768),
    ]


def draw(rng):
    """One more case of the same ranges: batches 1 to 64, a token to 32k, one new
    token to chunks of 2k, every head shape, both data types, paged and contiguous
    caches, whole, half and no rotation of a head, one to three axes of positions,
    one or two queries, windows or none."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    while True:
        c = dict(_BASE)
        c["op"] = rng.choice(["append", "append4", "read4", "attn4", "attn4"])
        c["heads"] = rng.choice(["28/4", "28/4", "28/4", "64/8", "32/8", "32/32", "16/16x64", "4/1x64"])
        hq, hkv, d = HEADS[c["heads"]]
        c["dtype"] = "f32" if rng.random() < 0.2 else "bf16"
        c["batch"] = log(1, 64)
        c["len_max"] = log(1, 32768)
        c["len_min"] = max(1, int(c["len_max"] * rng.choice([1.0, 0.6, 0.1])))
        c["room"] = rng.choice([0, 0, rng.randrange(1, 600)])
        c["page"] = rng.choice([0, 0, 16, 32, 128])
        c["mix"] = rng.randrange(1, 1 << 20)
        if c["op"] in ("append", "append4"):
            c["new_max"] = min(c["len_max"], log(1, 2048))
            c["new_min"] = rng.choice([0, 1, c["new_max"], max(1, c["new_max"] // 3)])
            c["rot"] = rng.choice([d, d, d, d // 2, 0])
            c["axes"] = rng.choice([0, 0, 1, 3])
            c["interleaved"] = rng.random() < 0.25
            c["fused"] = rng.random() < 0.7
        elif c["op"] == "attn4":
            c["sinks"] = rng.choice([0, 1, 4, 14, 37, 64])
            if rng.random() < 0.4:
                c["window"] = log(32, 8192)
            if 2 * hq // hkv <= 16 and rng.random() < 0.25:
                c["queries"] = 2
        # no larger than the largest listed case of the operator; caches of up to 512 MiB in 16 or 32 bits
        big = [work(x) for x in listed() if x["op"] == c["op"]]
        mine = work(c)
        rows = c["batch"] * _capacity(c) * hkv * d * 2
        if c["op"] != "attn4" and rows * _elem(c) > 1 << 29:
            continue
        if all(mine[k] <= max(b[k] for b in big) for k in mine):
            return c


# ---------------------------------------------------------------------------
# layout: a function of the case alone
# ---------------------------------------------------------------------------
def _lengths(case):
    r = random.Random(case["mix"])
    lens = [r.randint(case["len_min"], case["len_max"]) for _ in range(case["batch"])]
    lens[r.randrange(len(lens))] = case["len_max"]
    return lens


def _new(case):
    """New tokens of every sequence: its last ones."""
    r = random.Random(case["mix"] + 1)
    n = [r.randint(case["new_min"], case["new_max"]) for _ in range(case["batch"])]
    n[r.randrange(len(n))] = case["new_max"]
    return [min(a, b) for a, b in zip(n, _lengths(case))]


def _capacity(case):
    cap = case["len_max"] + case["room"]
    page = case["page"]
    return -(-cap // page) * page if page else cap


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows_read(case, n):
    """Rows of a sequence of n tokens that any of the queries sees."""
    if not case["window"]:
        return n
    lo = max(0, n - case["queries"] - case["window"] + 1)
    return n - max(0, lo - case["sinks"])


def _image(n):
    """An image's first row and side in a sequence of n tokens."""
    return min(14, n // 4), max(1, min(36, math.isqrt(n // 2)))


def _positions(case):
    """[axes][tokens] positions of the new tokens: an image's rows and columns
    count on two axes, everything else on all three together."""
    out = []
    for L, n in zip(_lengths(case), _new(case)):
        row = torch.arange(L - n, L)
        if case["axes"] < 3:
            out.append(row[None].expand(max(1, case["axes"]), n))
            continue
        at, side = _image(L)
        cell = row - at
        inside = (cell >= 0) & (cell < side * side)
        past = torch.where(cell >= side * side, row - side * side + side, row)
        out.append(torch.stack([torch.where(inside, torch.full_like(row, at), past),
                                torch.where(inside, at + cell.div(side, rounding_mode="floor"), past),
                                torch.where(inside, at + cell % side, past)]))
    return torch.cat(out, 1).to(torch.int32)


def _sections(case):
    """Frequency pairs of each axis: a quarter, three eighths, three eighths."""
    pairs = case["rot"] // 2
    if case["axes"] < 3:
        return [pairs] + [0] * 3
    first = max(4, pairs // 4 // 4 * 4)
    second = (pairs - first) // 8 * 4
    return [first, second, pairs - first - second, 0]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _generator(seed, salt):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 7919 + salt)
    return g


def _channels(case, g):
    """Widths of a KV head's channels: one in sixteen is six times the others."""
    _, hkv, d = HEADS[case["heads"]]
    return torch.where(torch.rand(hkv, 1, d, generator=g, device=DEVICE) < 1 / 16, 3.0, 0.5)


def _cos_sin(case):
    """[positions][rot]: cosines, then sines, of position / 1000000^(2 i / rot)."""
    rot = case["rot"]
    pos = torch.arange(_capacity(case) + 40, dtype=torch.float64)
    freq = 1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    a = pos[:, None] * freq
    return torch.cat([a.cos(), a.sin()], 1).float().to(DEVICE)


def _new_rows(case, seed):
    """q [n, Hq, d], k and v [n, Hkv, d] of the new tokens, as one product's columns or apart."""
    hq, hkv, d = HEADS[case["heads"]]
    n = sum(_new(case))
    g = _generator(seed, 29)
    x = torch.randn(n, hq + 2 * hkv, d, generator=g, device=DEVICE)
    x[:, hq:hq + hkv] *= _channels(case, g)[:, 0]
    x[:, hq + hkv:] *= 0.5
    x = x.to(_dtype(case))
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    return (q, k, v) if case["fused"] else (q.contiguous(), k.contiguous(), v.contiguous())


def _table(case, seed):
    """Where the blocks of the sequences lie: a random order, some blocks spare."""
    n = _capacity(case) // case["page"]
    total = case["batch"] * n + n // 2 + 1
    return torch.randperm(total, generator=_generator(seed, 5), device=DEVICE)[:case["batch"] * n], total


def _planes(case):
    """(blocks or sequences, rows of each) that a cache is made of."""
    if not case["page"]:
        return case["batch"], _capacity(case)
    n = _capacity(case) // case["page"]
    return case["batch"] * n + n // 2 + 1, case["page"]


def _old_rows(case, seed, which):
    """A cache of 16 or 32 bits as it is before the call."""
    _, hkv, d = HEADS[case["heads"]]
    n, rows = _planes(case)
    out = torch.empty(n, hkv, rows, d, dtype=_dtype(case), device=DEVICE)
    return out.normal_(0.0, 0.5, generator=_generator(seed, 31 + which))


def _query_rows(case, seed):
    """q [B, T, Hq, d] in 32 bits, and what an attended row adds to a key."""
    hq, hkv, d = HEADS[case["heads"]]
    B, T = case["batch"], case["queries"]
    q = torch.randn(B, T, hq, d, generator=_generator(seed, 41), device=DEVICE)
    q[:, 1:] = 0.9 * q[:, :1] + 0.43 * q[:, 1:]  # drafted queries follow the first one
    q0 = q[:, 0].reshape(B, hkv, hq // hkv, d)
    dirs = torch.nn.functional.normalize(q0.sum(2), dim=-1)
    proj = (q0 * dirs[:, :, None]).sum(-1).mean(2)
    return q, dirs * (SPIKE_NATS * math.sqrt(d) / proj)[..., None]


def _cached_rows(case, seed):
    """K and V of one sequence after another, [Hkv, length, d] in 32 bits."""
    _, hkv, d = HEADS[case["heads"]]
    _, step = _query_rows(case, seed)
    g = _generator(seed, 43)
    width = _channels(case, g)
    for b, L in enumerate(_lengths(case)):
        hit = torch.rand(L, generator=g, device=DEVICE) < 0.02
        K = torch.randn(hkv, L, d, generator=g, device=DEVICE).mul_(width)
        K.addcmul_(hit[None, :, None].float(), step[b, :, None])
        yield K, torch.randn(hkv, L, d, generator=g, device=DEVICE).mul_(0.5)


# ---------------------------------------------------------------------------
# 4 bits
# ---------------------------------------------------------------------------
_BYTES = {}


def _pairs_of_bytes():
    """float32 [256, 2]: the two elements of a byte, the low one first."""
    if "t" not in _BYTES:
        v = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])
        i = torch.arange(256)
        _BYTES["t"] = torch.stack([v[i % 16], v[i // 16]], 1).to(DEVICE)
    return _BYTES["t"]


def _to_4bit(x):
    """x [..., d] (32 or 64 bits) -> codes uint8 [..., d/2], scales uint8 [..., d/32]."""
    y = x.unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    e = torch.where(m > 0.875, e - 2, e - 3).clamp(-125, 125)
    e = torch.where(top == 0, -125, e)
    y = torch.ldexp(y.abs(), -e).unflatten(-1, (-1, 2))
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    code = code + 8 * torch.signbit(x.unflatten(-1, (-1, 32)).unflatten(-1, (-1, 2)))
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8).flatten(-2), (e + 127).to(torch.uint8).squeeze(-1)


def _from_4bit(codes, scales):
    """float32 [..., d] of codes and scales."""
    v = torch.index_select(_pairs_of_bytes(), 0, codes.reshape(-1).int()).view(*scales.shape, 32)
    return (v * torch.exp2(scales.float() - 127.0)[..., None]).flatten(-2)


def _round4(x):
    """The values that 4-bit rows hold of x [..., d], in 64 bits, from the numbers alone."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 7.0)))
    scale = torch.where(scale * 3.5 >= top, scale * 0.5, scale)  # (the logarithm's own rounding)
    scale = torch.where(scale * 7.0 < top, scale * 2.0, scale).clamp(2.0 ** -125, 2.0 ** 125)
    y = y / scale
    a = y.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)  # (round: to even)
    return (torch.copysign(a, y) * scale).flatten(-2)


# ---------------------------------------------------------------------------
# what a program has before the call
# ---------------------------------------------------------------------------
def _where(s, b, lo, hi):
    """(plane, row) of rows lo .. hi - 1 of sequence b."""
    pos = torch.arange(lo, hi, device=DEVICE)
    if s["table"] is None:
        return torch.full_like(pos, b), pos
    return s["table"][b].long()[pos // s["case"]["page"]], pos % s["case"]["page"]


def prepare(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    B, op = case["batch"], case["op"]
    i32 = dict(dtype=torch.int32, device=DEVICE)
    s = dict(case=case, op=op, table=None, seq_len=torch.tensor(_lengths(case), **i32))
    if case["page"]:
        s["table"] = _table(case, seed)[0].view(B, -1).to(torch.int32)
    if op in ("append", "append4"):
        s["q"], s["k"], s["v"] = _new_rows(case, seed)
        new = [0]
        for n in _new(case):
            new.append(new[-1] + n)
        s["new_off"] = torch.tensor(new, **i32)
        s["first"] = torch.tensor([a - b for a, b in zip(_lengths(case), _new(case))], **i32)
        s["pos"] = _positions(case).to(DEVICE)
        s["cos_sin"] = _cos_sin(case) if case["rot"] else None
        s["q_out"] = torch.zeros(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
    if op != "attn4":
        s["K"], s["V"] = _old_rows(case, seed, 0), _old_rows(case, seed, 1)
    if op != "append":
        n, rows = _planes(case)
        rows = -(-rows // 16) * 16
        for x in "kv":
            s[x + "4"] = (torch.zeros(n, hkv, rows, d // 2, dtype=torch.uint8, device=DEVICE),
                          torch.full((n, hkv, rows, d // 32), 127, dtype=torch.uint8, device=DEVICE))
    if op in ("read4", "attn4"):
        s["first"] = torch.zeros(B, **i32)
        for b, rows in enumerate(_cached_rows(case, seed)):
            at, row = _where(s, b, 0, rows[0].shape[1])
            for x, r in zip("kv", rows):
                for dst, src in zip(s[x + "4"], _to_4bit(r)):
                    dst[at, :, row] = src.transpose(0, 1)
    if op == "attn4":
        s["q"] = _query_rows(case, seed)[0].to(_dtype(case))
        s["out"] = torch.zeros(B * case["queries"], hq, d, dtype=s["q"].dtype, device=DEVICE)
    if own:
        _handle(s)
    return s


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _rotated(s, x):
    """x [n, H, d] rotated by the tokens' positions, in 64 bits (products of
    32-bit numbers are exact there)."""
    c, x = s["case"], x.double()
    rot = c["rot"]
    if not rot:
        return x
    axis = torch.repeat_interleave(torch.arange(4, device=DEVICE), torch.tensor(_sections(c), device=DEVICE))
    i = torch.arange(rot // 2, device=DEVICE)
    pos = s["pos"].long()[axis if c["axes"] == 3 else torch.zeros_like(axis)].T  # [n, pairs]
    cos = s["cos_sin"][pos, i].double()[:, None]
    sin = s["cos_sin"][pos, i + rot // 2].double()[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    lo, hi = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([lo, hi], -1).flatten(-2) if c["interleaved"] else torch.cat([lo, hi], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _new_places(s):
    """(plane, row) of every new token."""
    c = s["case"]
    lens, new = _lengths(c), _new(c)
    at = [_where(s, b, L - n, L) for b, (L, n) in enumerate(zip(lens, new))]
    return torch.cat([a for a, _ in at]), torch.cat([r for _, r in at])


def _plain_append(s):
    s["q_out"].copy_(_rotated(s, s["q"]))
    k, v = _rotated(s, s["k"]), s["v"]
    at, row = _new_places(s)
    if s["op"] == "append4":
        for x, r in (("k", k), ("v", v.double())):
            for dst, src in zip(s[x + "4"], _to_4bit(r)):
                dst[at, :, row] = src
        k, v = (_from_4bit(*(t[at, :, row] for t in s[x + "4"])) for x in "kv")
    s["K"][at, :, row] = k.to(s["K"].dtype)
    s["V"][at, :, row] = v.to(s["V"].dtype)
    return {"q": s["q_out"], "K": s["K"], "V": s["V"]}


def _plain_read(s):
    for b, L in enumerate(_lengths(s["case"])):
        at, row = _where(s, b, 0, L)
        for x, dst in (("k", s["K"]), ("v", s["V"])):
            dst[at, :, row] = _from_4bit(*(t[at, :, row] for t in s[x + "4"])).to(dst.dtype)
    return {"K": s["K"], "V": s["V"]}


def _plain_attention(s):
    c = s["case"]
    hq, hkv, d = HEADS[c["heads"]]
    B, T, W, S = c["batch"], c["queries"], c["window"], c["sinks"]
    G = hq // hkv
    q = s["q"].float().view(B, T, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, T * G, d)
    for b, L in enumerate(_lengths(c)):
        at, row = _where(s, b, 0, L)
        pos = torch.arange(L, device=DEVICE)
        if W and S + W + T - 1 < L:
            keep = (pos < S) | (pos > L - T - W)
            at, row, pos = at[keep], row[keep], pos[keep]
        K, V = (_from_4bit(*(t[at, :, row] for t in s[x + "4"])).transpose(0, 1) for x in "kv")
        p = L - T + torch.arange(T, device=DEVICE)  # the queries' positions
        see = pos <= p[:, None]
        if W:
            see = see & ((pos < S) | (pos > p[:, None] - W))  # [T, n]
        z = torch.matmul(q[b], K.transpose(1, 2).contiguous()) / math.sqrt(d)
        z = z.view(hkv, T, G, -1).masked_fill(~see[:, None], -math.inf)
        m = z.amax(-1, keepdim=True)
        w = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
        w = w / w.sum(-1, keepdim=True).clamp(min=1e-30)
        o = torch.matmul(w.view(hkv, T * G, -1), V.contiguous())
        s["out"][b * T:(b + 1) * T] = o.view(hkv, T, G, d).transpose(0, 1).reshape(T, hq, d)
    return {"out": s["out"]}


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _handle(s):
    """Shape, layout, options and workspace: made at a program's start and kept."""
    from paper_2605_31457_amd import vp
    c = s["case"]
    hq, hkv, d = HEADS[c["heads"]]
    cap = _capacity(c)
    sb, sh, ss = s["K"].stride()[:3] if "K" in s else (hkv * cap * d, cap * d, d)
    s["vp"] = vp
    s["shape"] = vp.vp_shape(
        batch=c["batch"], n_q_heads=hq, n_kv_heads=hkv, head_dim=d,
        dtype=vp.VP_BF16 if c["dtype"] == "bf16" else vp.VP_F32, max_seq_len=cap, max_vis=cap, max_segs=1, k_cap=cap,
        block_size=c["page"], scope=vp.VP_SCOPE_SEQUENCE, n_queries=c["queries"],
        kv_stride_b=sb, kv_stride_h=sh, kv_stride_s=ss)
    s["layout"] = vp.vp_layout(seq_len=s["seq_len"].data_ptr(), vis_seg_off=None, vis_seg=None,
                               block_table=None if s["table"] is None else s["table"].data_ptr())
    if c["op"] in ("append", "append4"):
        sec = _sections(c)
        s["rope"] = None if not c["rot"] else vp.vp_rope(
            cos_sin=s["cos_sin"].data_ptr(), n_pos=s["cos_sin"].shape[0], rot_dim=c["rot"],
            interleaved=int(c["interleaved"]), pos=None if c["axes"] == 0 else s["pos"].data_ptr(),
            n_axes=max(1, c["axes"]), section=(ctypes.c_int32 * 4)(*sec))
        s["tokens"] = vp.vp_tokens(
            q=s["q"].data_ptr(), k=s["k"].data_ptr(), v=s["v"].data_ptr(), q_stride=s["q"].stride(0),
            k_stride=s["k"].stride(0), v_stride=s["v"].stride(0), new_off=s["new_off"].data_ptr(),
            n_tokens=s["q"].shape[0])
    if c["op"] != "append":
        codes, scales = s["k4"]
        s["cache"] = vp.vp_kv4(
            k_codes=codes.data_ptr(), k_scales=scales.data_ptr(), v_codes=s["v4"][0].data_ptr(),
            v_scales=s["v4"][1].data_ptr(), code_stride_b=codes.stride(0), code_stride_h=codes.stride(1),
            scale_stride_b=scales.stride(0), scale_stride_h=scales.stride(1))
    if c["op"] == "attn4":
        s["options"] = vp.vp_window(window=c["window"], n_sink=c["sinks"], sm_scale=0.0)
        s["ws_bytes"] = vp.vp_kv4_workspace_size(s["shape"], s["options"])
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEVICE)


def _own(s):
    vp, op = s["vp"], s["op"]
    a = (s["shape"], s["layout"])
    if op == "attn4":
        vp.vp_kv4_decode_attn(*a, s["options"], s["q"], s["cache"], s["out"], s["ws"], s["ws_bytes"])
        return {"out": s["out"]}
    if op == "append":
        vp.vp_append_kv(*a, s["rope"], s["tokens"], s["q_out"], s["K"], s["V"])
        return {"q": s["q_out"], "K": s["K"], "V": s["V"]}
    if op == "append4":
        vp.vp_append_kv4(*a, s["rope"], s["tokens"], s["q_out"], s["cache"])
        vp.vp_kv4_read(*a, s["cache"], s["first"], s["K"], s["V"])
        return {"q": s["q_out"], "K": s["K"], "V": s["V"]}
    vp.vp_kv4_read(*a, s["cache"], None, s["K"], s["V"])
    return {"K": s["K"], "V": s["V"]}


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "append4": _plain_append, "read4": _plain_read, "attn4": _plain_attention}[s["op"]](s)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and how exact it is
# ---------------------------------------------------------------------------
def work(case):
    """Appending: the new rows of q, k and v read, the rotated queries and the cached
    rows written, a row of cosines and sines per position. Into 4 bits: codes and
    scales written, read back, and the rows written in 16 or 32 bits. Reading: codes
    and scales in, rows out. Attention: codes and scales of every row that a query
    sees, the queries and the outputs."""
    hq, hkv, d = HEADS[case["heads"]]
    e, T, op = _elem(case), case["queries"], case["op"]
    four = 2 * hkv * (d // 2 + d // 32)  # a token's keys and values in 4 bits
    nbytes = flops = 0
    for L, n in zip(_lengths(case), _new(case)):
        if op in ("append", "append4"):
            rows = n * (hq + 2 * hkv) * d * e
            nbytes += 2 * rows + 4 * n * case["rot"] + 4 * n * case["axes"]
            flops += 3 * n * (hq + hkv) * case["rot"]
            if op == "append4":
                nbytes += 2 * n * four
                flops += 4 * n * hkv * d
        elif op == "read4":
            nbytes += L * (four + 2 * hkv * d * e)
            flops += 2 * L * hkv * d
        else:
            rows = _rows_read(case, L)
            nbytes += rows * four + 2 * T * hq * d * e
            flops += 4 * T * hq * d * rows
    return {"bytes": nbytes, "flops": flops}


def _turned(case, x, pos, table):
    """x [n, H, d] as complex numbers times those of the positions."""
    rot = case["rot"]
    x = x.double()
    if not rot:
        return x
    sec = _sections(case)
    factor = []
    for axis in range(4):
        i = range(sum(sec[:axis]), sum(sec[:axis + 1]))
        if len(i):
            t = table[pos[axis if case["axes"] == 3 else 0].long()].double()
            factor.append(torch.complex(t[:, i.start:i.stop], t[:, rot // 2 + i.start:rot // 2 + i.stop]))
    factor = torch.cat(factor, 1)[:, None]
    pairs = x[..., :rot].unflatten(-1, (-1, 2)) if case["interleaved"] else x[..., :rot].unflatten(-1, (2, -1)).transpose(-1, -2)
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * factor)
    y = y if case["interleaved"] else y.transpose(-1, -2)
    return torch.cat([y.flatten(-2), x[..., rot:]], -1)


def exact(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    op, P = case["op"], case["page"]
    where = _table(case, seed)[0].view(case["batch"], -1).tolist() if P else None

    def put(cache, b, first, rows):
        """rows [n, Hkv, d] to rows first ... of sequence b."""
        n = rows.shape[0]
        while n:
            plane, row = (where[b][first // P], first % P) if P else (b, first)
            take = min(n, P - row) if P else n
            cache[plane, :, row:row + take] = rows[:take].transpose(0, 1)
            rows, first, n = rows[take:], first + take, n - take

    if op == "attn4":
        return _exact_attention(case, seed)
    K, V = (_old_rows(case, seed, i).double() for i in (0, 1))
    if op == "read4":
        for b, (k, v) in enumerate(_cached_rows(case, seed)):
            put(K, b, 0, _round4(k).transpose(0, 1))
            put(V, b, 0, _round4(v).transpose(0, 1))
        return {"K": K, "V": V}
    q, k, v = _new_rows(case, seed)
    pos = _positions(case).to(DEVICE)
    table = _cos_sin(case) if case["rot"] else None
    q, k, v = _turned(case, q, pos, table), _turned(case, k, pos, table), v.double()
    if op == "append4":
        k, v = _round4(k), _round4(v)
    i = 0
    for b, (L, n) in enumerate(zip(_lengths(case), _new(case))):
        put(K, b, L - n, k[i:i + n])
        put(V, b, L - n, v[i:i + n])
        i += n
    return {"q": q, "K": K, "V": V}


def _exact_attention(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    B, T, W, S = case["batch"], case["queries"], case["window"], case["sinks"]
    G = hq // hkv
    q = _query_rows(case, seed)[0].to(_dtype(case)).double()
    out = torch.zeros(B, T, hq, d, dtype=torch.float64, device=DEVICE)
    for b, (K, V) in enumerate(_cached_rows(case, seed)):
        n = K.shape[1]
        K, V = _round4(K), _round4(V)
        for t in range(T):
            at = n - T + t
            if at < 0:
                continue
            rows = torch.arange(at + 1, device=DEVICE)
            if W:
                rows = rows[(rows > at - W) | (rows < S)]
            A = torch.softmax(torch.matmul(K[:, rows], q[b, t].view(hkv, G, d).transpose(1, 2).contiguous()) * d ** -0.5, 1)
            out[b, t] = torch.matmul(A.transpose(1, 2).contiguous(), V[:, rows]).reshape(hq, d)
    return {"out": out.view(B * T, hq, d)}
