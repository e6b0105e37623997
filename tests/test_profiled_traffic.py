"""The benchmark reports the split kernel's DRAM traffic from the committed counters, as long as those were taken from
the kernel's present source."""
import pytest

import bench


def test_the_counters_are_those_of_the_present_source():
    traffic = bench.profiled_traffic("any", 2001920000)
    assert traffic == pytest.approx(2001920000, rel=0.02)          # every K and V byte once, and the partial results
    assert bench.profiled_traffic("any", 2 * 2001920000) == pytest.approx(2 * traffic)
