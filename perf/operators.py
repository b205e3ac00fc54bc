"""Decoding on a bounded cache, as measurable cases.

  op "window"  vp_window_decode_attn: attention of a step's queries over the
               window before them and the first tokens (sinks);
  op "sums"    the same call over the whole cache or a window, which also adds
               every row's attention weight to the running sums that eviction
               goes by;
  op "evict"   vp_evict: the rows of the largest sums, the first and the last
               ones stay, and the caches, sums and visual segments are
               compacted.

Lengths vary over the batch between `len_min` and `len_max` and depend on the
case alone (`mix`); `room` rows past the longest sequence are free. Keys and
values are Gaussian of scale 0.5; one row in fifty points along its KV group's
queries, so that attention is spread as unevenly as in a trained model.
Accumulated sums are log-normal: a few rows hold most of the weight.
"""
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

_BASE = dict(op="window", heads="28/4", dtype="bf16", batch=1, len_min=3358, len_max=3358, room=0, page=0, queries=1,
             window=0, sinks=4, budget=0, recent=0, kv_groups=False, images=1, mix=1)


def _case(name, **kw):
    c = dict(_BASE, name=name)
    for k, v in kw.items():
        assert k in c, k
        c[k] = v
    if "len_max" in kw and "len_min" not in kw:
        c["len_min"] = c["len_max"]
    return c


def listed():
    return [
        # window attention: the smallest call, one short fp32 sequence (a tiny
        # draft model's window layer); launches and dependent loads are all there is
        _case("win_tiny_f32", heads="4/1x64", dtype="f32", len_max=384, window=128),
        # one user's decode step in a window layer
        _case("win_b1_3k", window=1024),
        # a serving batch from a paged cache, two drafted queries per sequence,
        # sequences shorter than the window among them; the system text stays visible
        _case("win_b16_paged_q2", batch=16, len_min=500, len_max=12288, window=4096, sinks=14, page=32, queries=2, mix=3),
        # the largest: 64 long contexts, an 8k window
        _case("win_b64_32k", batch=64, len_max=32768, window=8192, sinks=64),
        # attention that leaves its weights: a short fp32 sequence
        _case("sum_tiny_f32", op="sums", heads="4/1x64", dtype="f32", len_max=384),
        # one KV head per query head, odd ragged lengths (older models)
        _case("sum_mha_b4", op="sums", heads="32/32", batch=4, len_min=1276, len_max=2477, mix=2),
        # 72B-class heads, paged in blocks of 16 rows, two queries
        _case("sum_b8_72b_paged", op="sums", heads="64/8", batch=8, len_min=6000, len_max=10753, page=16, queries=2,
              mix=5),
        # whole contexts of 32k tokens
        _case("sum_b16_32k", op="sums", batch=16, len_max=32768),
        # eviction: a short fp32 sequence
        _case("ev_tiny_f32", op="evict", heads="4/1x64", dtype="f32", len_max=384, budget=256, recent=64),
        # one user's cache back to half, every KV head its own rows
        _case("ev_b1_8k", op="evict", len_max=8192, budget=4096, recent=512, kv_groups=True),
        # a paged serving batch, one kept set per sequence and its images' segments;
        # short sequences stay whole
        _case("ev_b16_paged", op="evict", batch=16, len_min=5000, len_max=12288, budget=6144, sinks=14, recent=1024,
              page=32, images=2, room=96, mix=4),
        # the largest: 32 contexts of 32k tokens back to half
        _case("ev_b32_32k", op="evict", batch=32, len_max=32768, budget=16384, recent=2048, kv_groups=True),
    ]


def draw(rng):
    """One more case of the same ranges: batches 1 to 64, a hundred to 32k
    tokens, every head shape, both data types, paged and contiguous caches, one
    or two queries, windows and budgets from a few dozen rows to the whole cache."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    while True:
        c = dict(_BASE)
        c["op"] = rng.choice(["window", "sums", "evict"])
        c["heads"] = rng.choice(["28/4", "28/4", "28/4", "64/8", "32/8", "32/32", "16/16x64", "4/1x64"])
        c["dtype"] = "f32" if rng.random() < 0.15 else "bf16"
        c["batch"] = log(1, 64)
        c["len_max"] = log(100, 32768)
        c["len_min"] = max(1, int(c["len_max"] * rng.choice([1.0, 0.6, 0.1])))
        c["room"] = rng.choice([0, 0, rng.randrange(1, 600)])
        c["page"] = rng.choice([0, 0, 0, 16, 32, 128])
        c["sinks"] = rng.choice([0, 1, 4, 14, 37, 64])
        c["mix"] = rng.randrange(1, 1 << 20)
        hq, hkv, _ = HEADS[c["heads"]]
        if c["op"] == "evict":
            c["budget"] = max(c["sinks"] + 16, int(c["len_max"] * rng.uniform(0.25, 0.95)))
            c["recent"] = int((c["budget"] - c["sinks"]) * rng.uniform(0.0, 0.6))
            c["kv_groups"] = rng.random() < 0.5
            c["images"] = rng.choice([1, 2, 4])
            if c["budget"] >= c["len_max"]:
                continue
        else:
            if c["op"] == "window" or rng.random() < 0.3:
                c["window"] = log(32, 8192)
            if 2 * hq // hkv <= 16 and rng.random() < 0.25:
                c["queries"] = 2
        # no larger than the largest listed case of the operator; paged caches up
        # to 1 GiB of keys, as serving engines' pools are split
        big = [x for x in listed() if x["op"] == c["op"]][-1]
        most = 1 << 31 if c["page"] else _cache_bytes(big)
        mine, top = work(c), work(big)
        if _cache_bytes(c) <= most and all(mine[k] <= top[k] for k in mine):
            return c


# ---------------------------------------------------------------------------
# layout: a function of the case alone
# ---------------------------------------------------------------------------
def _lengths(case):
    r = random.Random(case["mix"])
    lens = [r.randint(case["len_min"], case["len_max"]) for _ in range(case["batch"])]
    lens[r.randrange(len(lens))] = case["len_max"]
    return lens


def _segments(case):
    """Per sequence `images` visual segments of an eighth of its rows each."""
    out = []
    for n in _lengths(case):
        part, size = n // case["images"], max(1, n // 8)
        out.append([(i * part + min(part // 4, 14), size) for i in range(case["images"])] if n >= 64 else [(0, 1)])
    return out


def _capacity(case):
    cap = case["len_max"] + case["room"]
    page = case["page"]
    return -(-cap // page) * page if page else cap


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def _cache_bytes(case):
    _, hkv, d = HEADS[case["heads"]]
    return 2 * case["batch"] * hkv * _capacity(case) * d * _elem(case)


def _rows_read(case, n):
    """Rows of a sequence of n tokens that any of the queries sees."""
    if not case["window"]:
        return n
    lo = max(0, n - case["queries"] - case["window"] + 1)
    return n - max(0, lo - case["sinks"])


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _inputs(case, seed):
    """q [B, T, Hq, d], K and V [B, Hkv, cap, d] and the sums [B, Hkv, cap]."""
    hq, hkv, d = HEADS[case["heads"]]
    B, T, cap = case["batch"], case["queries"], _capacity(case)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 7919 + 29)
    q = torch.randn(B, T, hq, d, generator=g, device=DEVICE)
    q[:, 1:] = 0.9 * q[:, :1] + 0.43 * q[:, 1:]  # drafted queries follow the first one
    q0 = q[:, 0].reshape(B, hkv, hq // hkv, d)
    dirs = torch.nn.functional.normalize(q0.sum(2), dim=-1)
    proj = (q0 * dirs[:, :, None]).sum(-1).mean(2)
    step = dirs * (SPIKE_NATS * math.sqrt(d) / proj)[..., None]
    K = torch.empty(B, hkv, cap, d, dtype=dt, device=DEVICE)
    V = torch.empty(B, hkv, cap, d, dtype=dt, device=DEVICE)
    for b in range(B):
        hit = torch.rand(cap, generator=g, device=DEVICE) < 0.02
        Kb = torch.randn(hkv, cap, d, generator=g, device=DEVICE).mul_(0.5)
        K[b] = torch.addcmul(Kb, hit[None, :, None].float(), step[b, :, None]).to(dt)
        V[b] = torch.randn(hkv, cap, d, generator=g, device=DEVICE).mul_(0.5).to(dt)
    sums = torch.randn(B, hkv, cap, generator=g, device=DEVICE).mul_(2.0).exp_().mul_(1e-3)
    return q.to(dt), K, V, sums


def _table(case, seed):
    """Where the blocks of the sequences lie: a random order, some blocks spare."""
    n = _capacity(case) // case["page"]
    total = case["batch"] * n + n // 2 + 1
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed) * 104729 + 5)
    return torch.randperm(total, generator=g, device=DEVICE)[:case["batch"] * n], total


def prepare(case, seed):
    hq, hkv, d = HEADS[case["heads"]]
    B, T, cap, P = case["batch"], case["queries"], _capacity(case), case["page"]
    q, K, V, sums = _inputs(case, seed)
    i32 = dict(dtype=torch.int32, device=DEVICE)
    table = None
    if P:
        where, total = _table(case, seed)

        def deal(x):
            out = torch.zeros(total, hkv, P, d, dtype=x.dtype, device=DEVICE)
            out[where] = x.view(B, hkv, cap // P, P, d).transpose(1, 2).reshape(-1, hkv, P, d)
            return out

        K, V, table = deal(K), deal(V), where.view(B, -1).to(torch.int32)
    off, flat = [0], []
    for s in _segments(case):
        flat += s
        off.append(len(flat))
    s = dict(op=case["op"], case=case, q=q, K=K, V=V, sums=sums, table=table,
             seq_len=torch.tensor(_lengths(case), **i32), off=torch.tensor(off, **i32), seg=torch.tensor(flat, **i32))
    if case["op"] == "evict":
        rows = B * (hkv if case["kv_groups"] else 1)
        s["kept"] = torch.full((rows, case["budget"]), -1, **i32)
        # the compacted sums, lengths and segments: buffers of their own, which
        # the program's next steps take up
        s["sums_out"] = torch.zeros_like(sums)
        s["seg_out"] = torch.zeros_like(s["seg"])
        s["new_len"] = torch.zeros(B, **i32)
    else:
        s["out"] = torch.zeros(B * T, hq, d, dtype=q.dtype, device=DEVICE)
    if own:
        _handle(s)
    return s


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------
def _rows(s, x, pos):
    """Cache rows at positions pos [B, n] as [B, Hkv, n, d] in 32 bits."""
    B = pos.shape[0]
    if s["table"] is None:
        b = torch.arange(B, device=DEVICE)[:, None]
        return x.transpose(1, 2)[b, pos].transpose(1, 2).float()
    P = s["case"]["page"]
    blk = torch.gather(s["table"].long(), 1, pos // P)
    return x[blk, :, pos % P].transpose(1, 2).float()


def _plain_attention(s):
    c = s["case"]
    hq, hkv, d = HEADS[c["heads"]]
    B, T, W, S = c["batch"], c["queries"], c["window"], c["sinks"]
    G, cap = hq // hkv, _capacity(c)
    L = s["seq_len"].long()
    p = L[:, None] - T + torch.arange(T, device=DEVICE)  # the queries' positions
    if W and S + W + T - 1 < cap:
        i = torch.arange(S + W + T - 1, device=DEVICE)
        first = (L - T - W + 1).clamp(min=S)  # the window's first row, past the sinks
        pos = torch.where(i < S, i, first[:, None] + i - S)
    else:
        pos = torch.arange(cap, device=DEVICE).expand(B, cap)
    see = (pos[:, None] <= p[..., None]) & (pos < L[:, None])[:, None]
    if W:
        see = see & ((pos[:, None] < S) | (pos[:, None] > p[..., None] - W))  # [B, T, n]
    at = pos.clamp(max=cap - 1)
    q = s["q"].float().view(B, T, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, T * G, d)
    z = torch.matmul(q, _rows(s, s["K"], at).transpose(2, 3).contiguous()) / math.sqrt(d)
    z = z.view(B, hkv, T, G, -1).masked_fill(~see[:, None, :, None], -math.inf)
    m = z.amax(-1, keepdim=True)
    w = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
    w = w / w.sum(-1, keepdim=True).clamp(min=1e-30)
    o = torch.matmul(w.view(B, hkv, T * G, -1), _rows(s, s["V"], at))
    o = o.view(B, hkv, T, G, d).permute(0, 2, 1, 3, 4).reshape(B * T, hq, d)
    s["out"].copy_(o)
    if s["op"] == "window":
        return {"out": s["out"]}
    add = torch.zeros(B, hkv, cap, device=DEVICE)
    add.scatter_add_(2, at[:, None].expand(B, hkv, -1), w.sum((2, 3)))  # rows past the end add zero
    here = torch.arange(cap, device=DEVICE)
    new = (here >= L[:, None] - T) & (here < L[:, None])
    s["sums"].copy_(torch.where(new[:, None], 0.0, s["sums"]) + add)
    return {"out": s["out"], "attn_sum": s["sums"]}


def _plain_evict(s):
    c = s["case"]
    hq, hkv, d = HEADS[c["heads"]]
    B, C, cap = c["batch"], c["budget"], _capacity(c)
    L = s["seq_len"].long()[:, None, None]
    here = torch.arange(cap, device=DEVICE)
    score = s["sums"] if c["kv_groups"] else s["sums"].double().sum(1, keepdim=True).float()
    score = score.masked_fill((here < c["sinks"]) | (here >= L - c["recent"]), math.inf).masked_fill(here >= L, -math.inf)
    kept = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :C].sort(-1)[0]
    live = kept < L  # rows past a short sequence's end sort last
    s["kept"].copy_(torch.where(live, kept, -1).view(-1, C))
    s["new_len"].copy_(live[:, 0].sum(-1))
    src = kept.expand(B, hkv, C)
    ok = live.expand(B, hkv, C)
    new = torch.arange(C, device=DEVICE)
    sums = torch.gather(s["sums"], 2, src)
    s["sums_out"][..., :C] = torch.where(ok, sums, s["sums_out"][..., :C])
    if s["table"] is None:
        at = src[..., None].expand(B, hkv, C, d)
        s["K"][:, :, :C] = torch.where(ok[..., None], torch.gather(s["K"], 2, at), s["K"][:, :, :C])
        s["V"][:, :, :C] = torch.where(ok[..., None], torch.gather(s["V"], 2, at), s["V"][:, :, :C])
    else:
        P, table = c["page"], s["table"].long()
        h = torch.arange(hkv, device=DEVICE)[None, :, None]
        blk = torch.gather(table[:, None].expand(B, hkv, -1), 2, src // P)
        to = table[:, None, new // P].expand(B, hkv, C)
        to_row = (new % P).expand(B, hkv, C)
        s["K"][to, h, to_row] = torch.where(ok[..., None], s["K"][blk, h, src % P], s["K"][to, h, to_row])
        s["V"][to, h, to_row] = torch.where(ok[..., None], s["V"][blk, h, src % P], s["V"][to, h, to_row])
    out = {"kept": s["kept"], "new_len": s["new_len"], "K": s["K"], "V": s["V"], "attn_sum": s["sums_out"]}
    if not c["kv_groups"]:
        seq = torch.repeat_interleave(torch.arange(B, device=DEVICE), (s["off"][1:] - s["off"][:-1]).long(),
                                      output_size=s["seg"].shape[0])
        rows = torch.where(live, kept, cap)[seq, 0]  # [segments, C]
        a, n = s["seg"][:, 0].long(), s["seg"][:, 1].long()
        start = (rows < a[:, None]).sum(-1)
        s["seg_out"].copy_(torch.stack([start, (rows < (a + n)[:, None]).sum(-1) - start], -1))
        out["vis_seg"] = s["seg_out"]
    return out


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _handle(s):
    """Shape, layout, options and workspace: made at a program's start and kept."""
    from paper_2605_31457_amd import vp
    c = s["case"]
    hq, hkv, d = HEADS[c["heads"]]
    sb, sh, ss, _ = s["K"].stride()
    s["vp"] = vp
    s["shape"] = vp.vp_shape(
        batch=c["batch"], n_q_heads=hq, n_kv_heads=hkv, head_dim=d,
        dtype=vp.VP_BF16 if c["dtype"] == "bf16" else vp.VP_F32, max_seq_len=_capacity(c), max_vis=_capacity(c),
        max_segs=c["images"], k_cap=_capacity(c), block_size=c["page"],
        scope=vp.VP_SCOPE_KV_GROUP if c["kv_groups"] else vp.VP_SCOPE_SEQUENCE, n_queries=c["queries"],
        kv_stride_b=sb, kv_stride_h=sh, kv_stride_s=ss)
    s["layout"] = vp.vp_layout(seq_len=s["seq_len"].data_ptr(), vis_seg_off=s["off"].data_ptr(),
                               vis_seg=s["seg"].data_ptr(),
                               block_table=None if s["table"] is None else s["table"].data_ptr())
    if s["op"] == "evict":
        s["options"] = vp.vp_evict_params(budget=c["budget"], n_sink=c["sinks"], n_recent=c["recent"])
        s["ws_bytes"] = vp.vp_evict_workspace_size(s["shape"], s["options"])
    else:
        s["options"] = vp.vp_window(window=c["window"], n_sink=c["sinks"], sm_scale=0.0)
        s["ws_bytes"] = vp.vp_window_workspace_size(s["shape"], s["options"], s["op"] == "sums")
    s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEVICE)


def _own(s):
    vp = s["vp"]
    a = (s["shape"], s["layout"], s["options"])
    if s["op"] == "evict":
        seg = None if s["case"]["kv_groups"] else s["seg_out"]
        vp.vp_evict(*a, s["sums"], s["K"], s["V"], s["kept"], s["sums_out"], seg, s["new_len"], s["ws"], s["ws_bytes"])
        out = {"kept": s["kept"], "new_len": s["new_len"], "K": s["K"], "V": s["V"], "attn_sum": s["sums_out"]}
        if seg is not None:
            out["vis_seg"] = seg
        return out
    sums = s["sums"] if s["op"] == "sums" else None
    vp.vp_window_decode_attn(*a, s["q"], s["K"], s["V"], sums, s["out"], s["ws"], s["ws_bytes"])
    return {"out": s["out"]} if sums is None else {"out": s["out"], "attn_sum": sums}


def run(s):
    if own:
        return _own(s)
    return _plain_evict(s) if s["op"] == "evict" else _plain_attention(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and how exact it is
# ---------------------------------------------------------------------------
def work(case):
    """Attention: the keys and values of every row that a query sees, the queries
    and outputs, and the sums of those rows read and written. Eviction: all sums
    read once, the kept rows past the sinks read and written, the kept lists and
    the compacted sums written."""
    hq, hkv, d = HEADS[case["heads"]]
    T, e = case["queries"], _elem(case)
    nbytes = flops = 0
    for n in _lengths(case):
        if case["op"] == "evict":
            C = case["budget"]
            nbytes += 4 * n * hkv + 4 * C * (hkv if case["kv_groups"] else 1) + 4 * min(n, C) * hkv
            if n > C:
                nbytes += 4 * (C - case["sinks"]) * hkv * d * e
                flops += n * hkv
        else:
            rows = _rows_read(case, n)
            nbytes += 2 * rows * hkv * d * e + 2 * T * hq * d * e
            flops += 4 * T * hq * d * rows
            if case["op"] == "sums":
                nbytes += 8 * rows * hkv
    return {"bytes": nbytes, "flops": flops}


def _exact_attention(case, q, K, V, sums):
    hq, hkv, d = HEADS[case["heads"]]
    B, T, W, S = case["batch"], case["queries"], case["window"], case["sinks"]
    G = hq // hkv
    out = torch.zeros(B, T, hq, d, dtype=torch.float64, device=DEVICE)
    sums = sums.double()
    for b, n in enumerate(_lengths(case)):
        sums[b, :, max(0, n - T):n] = 0.0
        for t in range(T):
            at = n - T + t
            if at < 0:
                continue
            rows = torch.arange(at + 1, device=DEVICE)
            if W:
                rows = rows[(rows > at - W) | (rows < S)]
            Kd = K[b][:, rows].double()
            Vd = V[b][:, rows].double()
            qd = q[b, t].double().view(hkv, G, d)
            A = torch.softmax(torch.matmul(Kd, qd.transpose(1, 2).contiguous()) * d ** -0.5, 1)  # [Hkv, n, G]
            out[b, t] = torch.matmul(A.transpose(1, 2).contiguous(), Vd).reshape(hq, d)
            sums[b][:, rows] += A.sum(-1)
    out = out.view(B * T, hq, d)
    return {"out": out} if case["op"] == "window" else {"out": out, "attn_sum": sums}


def _exact_evict(case, seed, K, V, sums):
    hq, hkv, d = HEADS[case["heads"]]
    B, C, S, R, P = case["batch"], case["budget"], case["sinks"], case["recent"], case["page"]
    U, cap = hkv if case["kv_groups"] else 1, _capacity(case)
    where, total = _table(case, seed) if P else (None, 0)
    kept = torch.full((B, U, C), -1, dtype=torch.int32, device=DEVICE)
    new_sums = torch.zeros(B, hkv, cap, dtype=torch.float64, device=DEVICE)
    new_len, segs = [], []
    for b, n in enumerate(_lengths(case)):
        new_len.append(min(n, C))
        for u in range(U):
            keep = list(range(n))
            if n > C:
                score = (sums[b, u] if case["kv_groups"] else sums[b].double().sum(0).float())[S:n - R].tolist()
                best = sorted(range(len(score)), key=lambda i: (-score[i], i))[:C - S - R]
                keep = list(range(S)) + sorted(S + i for i in best) + list(range(n - R, n))
            idx = torch.tensor(keep, device=DEVICE)
            kept[b, u, :len(keep)] = idx.to(torch.int32)
            heads = [u] if case["kv_groups"] else range(hkv)
            for g in heads:
                new_sums[b, g, :len(keep)] = sums[b, g, idx].double()
                K[b, g, :len(keep)] = K[b, g, idx].clone()
                V[b, g, :len(keep)] = V[b, g, idx].clone()
            if U == 1:
                for a, k in _segments(case)[b]:
                    before = sum(1 for x in keep if x < a)
                    segs.append((before, sum(1 for x in keep if x < a + k) - before))
    if P:
        def deal(x):
            out = torch.zeros(total, hkv, P, d, dtype=x.dtype, device=DEVICE)
            out[where] = x.view(B, hkv, cap // P, P, d).transpose(1, 2).reshape(-1, hkv, P, d)
            return out

        K, V = deal(K), deal(V)
    out = {"kept": kept.view(B * U, C), "new_len": torch.tensor(new_len, dtype=torch.int32), "K": K, "V": V,
           "attn_sum": new_sums}
    if U == 1:
        out["vis_seg"] = torch.tensor(segs, dtype=torch.int32)
    return out


def exact(case, seed):
    q, K, V, sums = _inputs(case, seed)
    if case["op"] == "evict":
        return _exact_evict(case, seed, K, V, sums)
    return _exact_attention(case, q, K, V, sums)
