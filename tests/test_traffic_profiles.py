"""The committed HBM traffic of the convolution kernels belongs to the committed sources: the benchmark
reports a figure only while its kernel's sources hash to the value recorded with it."""
import pytest

import bench


@pytest.mark.parametrize("key", sorted(bench.TRAFFIC_PROFILES))
def test_profile_is_of_these_sources(key):
    assert bench.committed_traffic(*key) is not None
