"""A program that keeps a layer's cache in 16 or 32 bits and another's in 4, as it would run:
prompts with images appended in chunks, decode steps that append and attend, rows read back for
the method's decode step, and the same captured in a graph."""
import numpy as np
import pytest
import torch

from _cache import assert_attention
from _kv4 import assert_rounded, attention_bound, cos_sin
from _parity import small_workload
from oracle import cache_oracle as CO
from oracle import kv4_oracle as KO
from oracle import vp_oracle as O
from paper_2605_31457_amd import step as S
from paper_2605_31457_amd import workloads as W

pytestmark = pytest.mark.gpu


def _tokens(g, n, Hq, Hkv, d, dtype):
    """A product's columns [n, Hq + 2 Hkv, d] on the device, and q, k, v in float64."""
    x = torch.from_numpy(g.standard_normal((n, Hq + 2 * Hkv, d))).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    f = x.double().numpy()
    x = x.cuda()
    return (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]), (f[:, :Hq], f[:, Hq:Hq + Hkv], f[:, Hq + Hkv:])


def _rows(ds, x, b, L):
    """Rows [Hkv, L, d] of sequence b in float64."""
    if ds.block_table is None:
        return x[b, :, :L].double().cpu().numpy()
    t = ds.block_table[b].long()
    return x[t].transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :L].double().cpu().numpy()


def _held(x):
    return KO.decode(*KO.quantise(x))


@pytest.mark.parametrize("dtype,T,block,d", [("bf16", 1, 0, 128), ("bf16", 2, 16, 64), ("f32", 1, 32, 64)])
def test_prompt_and_decode(dtype, T, block, d):
    B, Hq, Hkv, cap = 3, 8, 2, 256
    lens = [150, 40, 97]
    segs = [[(5, 60)], [], [(20, 30), (60, 20)]]
    w = small_workload(31, B, Hq, Hkv, d, lens, segs, dtype=dtype, S_cap=cap)
    if T > 1:
        w.q = np.repeat(w.q[:, None], T, 1)
    ds = S.DeviceStep(w, block_size=block)
    ds.make_kv4()
    g = np.random.default_rng(5)
    table = cos_sin(cap, d, 1)
    t = torch.from_numpy(table).cuda()
    sections = (d // 8, d // 8, d // 4)
    K, V = [np.zeros((Hkv, 0, d))] * B, [np.zeros((Hkv, 0, d))] * B  # unrounded rotated keys, values
    # the prompts, in two ragged chunks
    done = [0] * B
    for chunk in ([100, 40, 30], [50, 0, 67]):
        n = sum(chunk)
        dev, (q, k, v) = _tokens(g, n, Hq, Hkv, d, dtype)
        pos = g.integers(0, cap, (3, n))
        off = np.concatenate([[0], np.cumsum(chunk)])
        done = [a + c for a, c in zip(done, chunk)]
        ds.seq_len.copy_(torch.tensor(done, dtype=torch.int32))
        r = S.make_rope(t, torch.from_numpy(pos.astype(np.int32)).cuda(), sections)
        new_off = torch.from_numpy(off.astype(np.int32)).cuda()
        q_out = torch.zeros(n, Hq, d, dtype=ds.q.dtype, device=ds.device)
        assert ds.append(dev[1], dev[2], dev[0], r, new_off, q_out) is q_out
        kr = KO.rotate(k, table, pos, d, sections)
        assert_rounded(q_out.double().cpu().numpy(), KO.rotate(q, table, pos, d, sections), dtype)
        ds.append(dev[1], dev[2], rope=r, new_off=new_off, four=True)
        for b in range(B):
            K[b] = np.concatenate([K[b], kr[off[b]:off[b + 1]].transpose(1, 0, 2)], 1)
            V[b] = np.concatenate([V[b], v[off[b]:off[b + 1]].transpose(1, 0, 2)], 1)
    rope = S.make_rope(t)
    for step in range(12):
        dev, (q, k, v) = _tokens(g, B * T, Hq, Hkv, d, dtype)
        ds.seq_len.add_(T)
        done = [a + T for a in done]
        pos = np.concatenate([np.arange(L - T, L) for L in done])[None]
        ds.append(dev[1], dev[2], dev[0], rope)
        ds.append(dev[1], dev[2], rope=rope, four=True)
        kr = KO.rotate(k, table, pos, d)
        qs = ds.q.double().cpu().numpy().reshape(B, T, Hq, d)
        assert_rounded(qs.reshape(B * T, Hq, d), KO.rotate(q, table, pos, d), dtype)
        for b in range(B):
            K[b] = np.concatenate([K[b], kr[b * T:(b + 1) * T].transpose(1, 0, 2)], 1)
            V[b] = np.concatenate([V[b], v[b * T:(b + 1) * T].transpose(1, 0, 2)], 1)
        for window, four in ((0, False), (0, True), (70, True)):
            (ds.kv4_decode_attn if four else ds.window_decode_attn)(window, 4)
            out = ds.out.view(B, T, Hq, d)
            for b, L in enumerate(done):
                if four:
                    r = CO.window_attention(qs[b], _held(K[b]), _held(V[b]), window, 4)
                    bound = attention_bound(r, dtype, L, d, T * Hq)
                    assert np.all(np.abs(out[b].double().cpu().numpy() - r.out) <= bound), (step, b, window)
                else:
                    r = CO.window_attention(qs[b], _rows(ds, ds.K, b, L), _rows(ds, ds.V, b, L), window, 4)
                    assert_attention(out[b], r, dtype, L, f"step {step} seq {b}")
    for b, L in enumerate(done):
        assert_rounded(_rows(ds, ds.K, b, L), K[b], dtype)
        assert np.array_equal(_rows(ds, ds.V, b, L), V[b])
    if T > 1:
        return
    # the 4-bit rows back, and the method's step on them
    ds.kv4_read()
    stored = lambda x: x.astype(np.float32) if dtype == "f32" else W.bf16_round(x.astype(np.float32))
    Kh, Vh = (np.zeros((B, Hkv, cap, d)) for _ in range(2))
    for b, L in enumerate(done):
        Kh[b, :, :L], Vh[b, :, :L] = _held(K[b]), _held(V[b])
        assert np.array_equal(_rows(ds, ds.K, b, L), Kh[b, :, :L]) and np.array_equal(_rows(ds, ds.V, b, L), Vh[b, :, :L])
    w2 = W.Workload(name="read back", dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, d=d, S_cap=cap, seq_len=np.array(done, np.int32),
                    segments=segs, q=stored(ds.q.double().cpu().numpy().reshape(B, Hq, d)), K=stored(Kh), V=stored(Vh),
                    tau_mass=w.tau_mass, r_lo_bp=w.r_lo_bp, r_hi_bp=w.r_hi_bp, clamp=w.clamp)
    d2 = S.DeviceStep(w2, block_size=block, k_cap=ds.k_cap, max_vis=ds.max_vis)
    ds.vis_idx.fill_(-7)
    ds.decode_step()
    d2.decode_step()
    got, want = ds.results(), d2.results()
    for key in ("mass_head", "mass_seq", "k", "vis_idx", "out"):
        assert np.array_equal(got[key], want[key]), key


@pytest.mark.parametrize("block", [0, 16])
def test_step_captured_in_a_graph(block):
    """Lengths, both appends, attention over 4 bits and reading back in one graph, replayed with other tokens
    and eager work between, against the same calls made eagerly. Two graphs share the workspace."""
    B, Hq, Hkv, d, cap = 3, 28, 4, 128, 2048
    lens = [1500, 3, 700]
    w = small_workload(9, B, Hq, Hkv, d, lens, [[], [], []], S_cap=cap)
    t = torch.from_numpy(cos_sin(cap, d)).cuda()
    runs = []
    for captured in (False, True):
        g = np.random.default_rng(3)
        ds = S.DeviceStep(w, block_size=block, max_vis=1)
        ds.make_kv4()
        for x in ds.kv4_codes:
            x.random_(0, 256, generator=torch.Generator(device=ds.device).manual_seed(1))
        for x in ds.kv4_scales:
            x.fill_(127)
        (q, k, v), _ = _tokens(g, B, Hq, Hkv, d, "bf16")
        fresh = q.new_empty(B, Hq + 2 * Hkv, d)
        q, k, v = fresh[:, :Hq], fresh[:, Hq:Hq + Hkv], fresh[:, Hq + Hkv:]
        rope = S.make_rope(t)
        first = torch.zeros(B, dtype=torch.int32, device=ds.device)

        def step(window):
            torch.sub(ds.seq_len.add_(1), 1, out=first)
            ds.append(k, v, q, rope)
            ds.append(k, v, rope=rope, four=True)
            ds.kv4_decode_attn(window, 4)
            ds.kv4_read(first)

        fresh.zero_()
        for window in (0, 1024):  # (allocates)
            step(window)
        ds.seq_len.sub_(2)
        torch.cuda.synchronize()
        calls = [lambda: step(0), lambda: step(1024)]
        if captured:
            graphs = []
            for f in calls:
                graphs.append(torch.cuda.CUDAGraph())
                with torch.cuda.graph(graphs[-1]):
                    f()
            calls = [x.replay for x in graphs]
        log = []
        for rep in range(4):
            for f in calls:
                fresh.copy_(_tokens(g, B, Hq + 2 * Hkv, 0, d, "bf16")[0][0])
                f()
                torch.cuda.synchronize()
                log += [ds.out.clone(), ds.q.clone(), ds.seq_len.clone()]
                ds.out.zero_()
        log += [ds.K, ds.V, *ds.kv4_codes, *ds.kv4_scales]
        runs.append(log)
    for i, (x, y) in enumerate(zip(*runs)):
        assert torch.equal(x, y), i
    assert runs[0][0].abs().sum() > 0


def test_arguments():
    ds = S.DeviceStep(small_workload(5, 2, 4, 1, 64, [50, 20], [[], []]), max_vis=1)
    k = torch.zeros(2, 1, 64, dtype=torch.bfloat16, device=ds.device)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device=ds.device)
    t = torch.zeros(64, 64, device=ds.device)
    for call in (ds.kv4_decode_attn, ds.kv4_read, lambda: ds.append(k, k, four=True)):
        with pytest.raises(RuntimeError):
            call()
    for args in ((k.float(), k), (k, k[:1]), (k, k, q[:, :2]), (k, torch.zeros(2, 1, 128, dtype=k.dtype, device=k.device)[..., ::2]),
                 (k.cpu(), k.cpu())):
        with pytest.raises(ValueError):
            ds.append(*args)
    for kw in (dict(new_off=torch.zeros(2, dtype=torch.int32, device=ds.device)), dict(new_off=torch.zeros(3, device=ds.device)),
               dict(q_out=q), dict(q=q, q_out=q[:1]), dict(q=q, q_out=q.float()),
               dict(rope=S.make_rope(t, torch.zeros(5, dtype=torch.int32, device=ds.device)))):
        with pytest.raises(ValueError):
            ds.append(k, k, **kw)
    for a in ((t.double(),), (t[:, ::2],), (t, torch.zeros(2, device=ds.device)), (t, torch.zeros(2, dtype=torch.int32)),
              (t, torch.zeros(2, 2, dtype=torch.int32, device=ds.device)), (t, torch.zeros(2, dtype=torch.int32, device=ds.device), (16, 16)),
              (t, None, (4,) * 5)):
        with pytest.raises(ValueError):
            S.make_rope(*a)
    ds.make_kv4()
    with pytest.raises(ValueError):
        ds.kv4_read(torch.zeros(2, dtype=torch.int64, device=ds.device))
