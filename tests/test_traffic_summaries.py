"""The committed traffic summaries belong to the committed kernel sources: bench.py reports their bytes only then."""
import glob
import json
import os

import pytest

import bench

SUMMARIES = sorted(glob.glob(os.path.join(bench.ROOT, "profiles", "traffic_*.json")))


def test_every_workload_of_the_default_run_has_one():
    assert len(SUMMARIES) == 5


@pytest.mark.parametrize("path", SUMMARIES, ids=os.path.basename)
def test_bench_reports_the_measured_bytes(path):
    key = os.path.basename(path)[len("traffic_"):-len(".json")]
    with open(path) as f:
        assert bench.measured_traffic(key) == json.load(f)["hbm_bytes_per_launch"]
