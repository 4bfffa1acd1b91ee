"""The benchmark's measured traffic: summaries under profiles/ that belong to the streaming kernel as it is (no GPU)."""

import pytest

import bench


@pytest.mark.parametrize("workload", ["lstm", "resnet50", "speech"])
def test_summary_of_this_kernel(workload):
    """Other kernels' sources may change without it."""
    names = bench.stream_sources()
    assert "dgc_compress.hip" in names and "dgc_internal.h" in names and "dgc_vocab.hip" not in names
    assert bench.measured_traffic(workload) is not None
