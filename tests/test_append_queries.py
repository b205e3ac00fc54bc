"""DeviceStep.append: where rotated queries go, and calls without tokens (no GPU)."""
import pytest
import torch

from paper_2605_31457_amd import step as S
from paper_2605_31457_amd import vp
from _parity import small_workload

B, HQ, HKV, D = 2, 4, 1, 64


@pytest.fixture
def calls(monkeypatch):
    """(step, the q_out of every call that reaches the library, with its number of tokens)"""
    ds = S.DeviceStep(small_workload(5, B, HQ, HKV, D, [50, 20], [[], []]), device="cpu", max_vis=1)
    ds.make_kv4()
    seen = []
    for name in ("vp_append_kv", "vp_append_kv4"):
        monkeypatch.setattr(vp, name, lambda shape, layout, rope, tokens, q_out, *a: seen.append((q_out, tokens.n_tokens)))
    monkeypatch.setattr(vp, "_on_current_device", lambda *a: None)
    return ds, seen


def _tokens(n):
    return [torch.zeros(n, H, D, dtype=torch.bfloat16) for H in (HKV, HKV, HQ)]


@pytest.mark.parametrize("four", [False, True])
def test_ragged_queries_need_a_place_of_their_own(calls, four):
    """As many tokens as the step has queries, but both of sequence 0: in `q` the second would be
    sequence 1's query."""
    ds, seen = calls
    k, v, q = _tokens(B)
    off = torch.tensor([0, 2, 2], dtype=torch.int32)
    with pytest.raises(ValueError, match="q_out"):
        ds.append(k, v, q, new_off=off, four=four)
    assert seen == []
    out = torch.zeros(B, HQ, D, dtype=torch.bfloat16)
    assert ds.append(k, v, q, new_off=off, q_out=out, four=four) is out
    assert ds.append(k, v, q, new_off=off, q_out=ds.q, four=four) is ds.q  # (the caller knows: one token each)
    assert ds.append(k, v, q, four=four) is ds.q
    assert ds.append(k, v, new_off=off, four=four) is None
    assert [x for x, _ in seen] == [out, ds.q, ds.q, None]


@pytest.mark.parametrize("four", [False, True])
def test_no_tokens(calls, four):
    """None at all, with and without queries, as the C calls take it: nothing is rotated."""
    ds, seen = calls
    k, v, q = _tokens(0)
    off = torch.zeros(B + 1, dtype=torch.int32)
    ds.append(k, v, q, new_off=off, four=four)
    ds.append(k, v, q, new_off=off, q_out=q.clone(), four=four)
    ds.append(k, v, new_off=off, four=four)
    assert [n for _, n in seen] == [0, 0, 0]
