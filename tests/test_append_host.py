"""DeviceStep.append before anything is enqueued (no GPU): what it refuses and what it passes on."""
import pytest
import torch

from paper_2605_31457_amd import step as S
from paper_2605_31457_amd import vp
from _parity import small_workload


def _step(Hkv=1, device="cpu"):
    return S.DeviceStep(small_workload(5, 2, 4, Hkv, 64, [50, 20], [[], []]), device=device, max_vis=1)


def test_rope_on_another_device():
    ds = _step(device="meta")
    k = torch.zeros(2, 1, 64, dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match="cos_sin"):
        ds.append(k, k, rope=S.make_rope(torch.zeros(64, 64)))


@pytest.mark.parametrize("four", [False, True])
def test_another_current_device(four, monkeypatch):
    ds = _step()
    ds.make_kv4()
    monkeypatch.setattr(vp, "_current_device", lambda: 0)  # (the buffers are on none)
    monkeypatch.setattr(vp, "_stream", lambda s: 0)
    k = torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        ds.append(k, k, four=four)


def test_one_head_of_any_stride(monkeypatch):
    """With one KV head the stride between heads means nothing."""
    ds = _step()
    seen = []
    monkeypatch.setattr(vp, "vp_append_kv", lambda shape, layout, rope, tokens, *a: seen.append((tokens.k_stride, tokens.v_stride)))
    x = torch.zeros(2, 256, dtype=torch.bfloat16)
    k, v = x[:, 64:128].as_strided((2, 1, 64), (256, 8, 1), 64), torch.zeros(1, 2, 64, dtype=torch.bfloat16).transpose(0, 1)
    ds.append(k, v)
    assert seen == [(256, 64)]
    with pytest.raises(ValueError, match="next to each other"):
        _step(Hkv=2).append(torch.zeros(2, 64, 2, dtype=torch.bfloat16).transpose(1, 2), torch.zeros(2, 2, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="next to each other"):
        ds.append(torch.zeros(2, 1, 128, dtype=torch.bfloat16)[..., ::2], v)
