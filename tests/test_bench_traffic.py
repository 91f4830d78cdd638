"""bench.py reports DRAM bytes per launch from the committed captures as long as the
kernels' code is what was captured."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
import bench  # noqa: E402


@pytest.mark.parametrize("kernel, profile", [
    ("verify_attention_kernel", bench.PROFILES["image7b"]), ("verify_attention_tc_kernel", bench.PROFILES["video"]),
    ("lm_head_kernel", bench.LM_HEAD_PROFILES["image7b"]), ("lm_head_kernel", bench.LM_HEAD_PROFILES["long"])])
def test_the_captures_are_of_the_kernels_that_are_built(kernel, profile):
    assert bench.profiled_traffic(bench.KERNEL_SOURCES[kernel], profile) is not None
