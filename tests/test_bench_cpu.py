"""CPU checks of what bench.py reports beside its timed figures."""
import pytest

import bench


@pytest.mark.parametrize("cfg", [4, 5])
def test_counted_traffic_belongs_to_the_present_kernels(cfg):
    """The committed counters were taken from the expert FFN kernels as they stand (else bench.py reports none)."""
    traffic, source = bench.measured_traffic(cfg)
    assert traffic is not None, source
