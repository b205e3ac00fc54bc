"""DeviceStep.make_kv4 over blocks that a 4-bit cache cannot have (no GPU)."""
import pytest

from paper_2605_31457_amd import step as S
from _parity import small_workload


def _step(block):
    return S.DeviceStep(small_workload(5, 2, 4, 1, 64, [50, 20], [[], []]), device="cpu", max_vis=1, block_size=block)


@pytest.mark.parametrize("block", [1, 2, 4, 8])
def test_refused(block):
    ds = _step(block)
    with pytest.raises(ValueError, match="16 rows"):
        ds.make_kv4()
    assert ds.kv4 is None


@pytest.mark.parametrize("block", [0, 16, 32])
def test_taken(block):
    ds = _step(block)
    assert ds.make_kv4() is ds.kv4
