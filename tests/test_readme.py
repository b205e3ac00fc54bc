"""README's programs that append, run with the library's calls replaced by a record of which rows
they set and read (no GPU)."""
import os
import re

import pytest
import torch

from conftest import ROOT
from paper_2605_31457_amd import step as S
from paper_2605_31457_amd import vp
from _parity import small_workload


def _programs():
    with open(os.path.join(ROOT, "README.md"), encoding="utf-8") as f:
        return [x for x in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "append(" in x]


class Record:
    """Rows of each sequence that are set, in the 16- and in the 4-bit cache."""

    def __init__(self, monkeypatch, ds):
        self.ds, self.wide, self.four = ds, [set(range(n)) for n in ds.seq_len.tolist()], [set() for _ in range(ds.w.B)]
        self.read = 0  # calls that attended over a cache or brought rows back
        for name in ("vp_append_kv", "vp_append_kv4", "vp_window_decode_attn", "vp_decode_step", "vp_kv4_decode_attn", "vp_kv4_read"):
            monkeypatch.setattr(vp, name, getattr(self, name))
        monkeypatch.setattr(vp, "_on_current_device", lambda *a: None)

    def _put(self, rows, tokens):
        lens, n = self.ds.seq_len.tolist(), tokens.n_tokens
        off = torch.tensor([n // len(lens) * b for b in range(len(lens) + 1)])
        if tokens.new_off:
            off = self.ns["new_off"]
            assert tokens.new_off == off.data_ptr()
        for b, L in enumerate(lens):
            count = int(off[b + 1] - off[b])
            assert 0 <= L - count and L <= self.ds.w.S_cap
            rows[b] |= set(range(L - count, L))

    def _whole(self, rows, first=None):
        self.read += 1
        for b, L in enumerate(self.ds.seq_len.tolist()):
            lo = 0 if first is None else int(first[b])
            assert rows[b] >= set(range(lo, L)), f"sequence {b}: rows that nothing has set are read"

    def vp_append_kv(self, shape, layout, rope, tokens, *a):
        self._put(self.wide, tokens)

    def vp_append_kv4(self, shape, layout, rope, tokens, *a):
        self._put(self.four, tokens)

    def vp_window_decode_attn(self, *a):
        self._whole(self.wide)

    def vp_decode_step(self, *a):
        self._whole(self.wide)

    def vp_kv4_decode_attn(self, *a):
        self._whole(self.four)

    def vp_kv4_read(self, shape, layout, cache, first, *a):
        self._whole(self.four, first)


@pytest.mark.parametrize("program", _programs(), ids=lambda x: "4 bits" if "make_kv4" in x else "16 bits")
def test_programs_read_what_they_have_set(program, monkeypatch):
    B, Hq, Hkv, d = 2, 4, 2, 64
    ds = S.DeviceStep(small_workload(5, B, Hq, Hkv, d, [20, 9], [[], []], S_cap=64), device="cpu", max_vis=1)
    r = Record(monkeypatch, ds)
    x = lambda n, H: torch.zeros(n, H, d, dtype=torch.bfloat16)
    r.ns = dict(step=S, torch=torch, ds=ds, cos_sin=torch.zeros(64, d), q=x(B, Hq), k=x(B, Hkv), v=x(B, Hkv),
                prompt_q=x(29, Hq), prompt_k=x(29, Hkv), prompt_v=x(29, Hkv), rotated=x(29, Hq),
                new_off=torch.tensor([0, 20, 29], dtype=torch.int32), prompt_len=torch.tensor([20, 9], dtype=torch.int32))
    exec(program, r.ns)
    assert r.read


def test_there_are_programs():
    assert any("make_kv4" in x for x in _programs())
