"""The committed ncu summaries of the forward kernel belong to its current source (host only): bench.py reports their
DRAM bytes, half of its metric, only as long as they do.  A helper that other kernels need goes into a file of theirs."""
import os
import re

import pytest

import bench


@pytest.mark.parametrize("workload", sorted(bench.PROFILES))
def test_summary_belongs_to_the_current_source(workload):
    with open(bench.PROFILES[workload]) as f:
        text = f.read()
    assert re.search(r"kernel_source_sha256:\s*([0-9a-f]{64})", text).group(1) == bench.kernel_source_hash()
    traffic = bench.profiled_traffic(workload)
    assert traffic["read"] > 0 and traffic["write"] >= 0


def test_every_summary_of_the_forward_kernel_is_current():
    folder = os.path.join(bench.ROOT, "profiles")
    found = 0
    for name in sorted(os.listdir(folder)):
        with open(os.path.join(folder, name)) as f:
            m = re.search(r"kernel_source_sha256:\s*([0-9a-f]{64})", f.read())
        if m:
            found += 1
            assert m.group(1) == bench.kernel_source_hash(), name
    assert found >= len(bench.PROFILES)
