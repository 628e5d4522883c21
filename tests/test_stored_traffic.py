"""The stored DRAM traffic that the bench line reports applies to the kernels
as they are: bench.py leaves a figure out where a kernel's sources have
changed since it was captured."""
import json
import os

import pytest

import bench

with open(os.path.join(bench.ROOT, "profiles", "traffic.json")) as f:
    STORED = {k: v for k, v in json.load(f).items() if isinstance(v, dict)}


@pytest.mark.parametrize("kernel", sorted(STORED))
def test_stored_traffic_applies(kernel):
    assert kernel in bench.TRAFFIC_SOURCES
    for workload, nbytes in STORED[kernel].items():
        if workload != "sha":
            assert bench._traffic(workload, kernel) == nbytes
