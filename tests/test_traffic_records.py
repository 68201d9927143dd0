"""The traffic records that the bench prices its roofline with hold only while their kernels' sources are unchanged."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

pytest.importorskip("torch")
import bench  # noqa: E402
import scram_inputs as si  # noqa: E402


@pytest.mark.parametrize("kernel", sorted(bench.KERNEL_SRCS))
@pytest.mark.parametrize("workload", ["self256_bf16", "large2048_bf16"])
def test_the_records_are_of_the_present_sources(workload, kernel):
    record = bench.load_traffic(si.get(workload), kernel)
    assert record is not None, f"profiles/traffic.json has no record of {kernel} as it is now: {bench.kernel_source_hash(kernel)}"
    assert record["bytes_per_launch"] > 0
