"""The kernels of a bounded cache keep what they hold in registers (no GPU)."""
import pytest

from tests.test_resources import resources


@pytest.mark.parametrize("source,kernels", [("kv_weigh.hip", 44), ("kv_evict.hip", 17)])
def test_nothing_spills(source, kernels):
    found = resources(source)
    assert len(found) == kernels
    for name, r in found.items():
        assert r["VGPRs Spill"] == 0 and r["ScratchSize"] == 0, (name, r)
