"""The DRAM traffic that the benchmark reports is on file for the loss kernels as they are (no GPU needed)."""
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import bench  # noqa: E402


@pytest.mark.parametrize("kernel", ["e", "dh", "dw"])
@pytest.mark.parametrize("d", [4096, 1024])
def test_counters_on_file_are_those_of_the_present_kernels(d, kernel):
    """A change of the loss kernels' code, and of no other, asks for a new capture."""
    moved, source = bench.dram_traffic(kernel, d, 151936, 8192)
    # the operands once at least: the weights in bfloat16
    assert moved is not None and moved > 2 * d * 151936, source
