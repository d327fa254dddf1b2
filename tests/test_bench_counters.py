"""The counter figures that bench.py reports beside its times belong to the
kernel sources in the tree: a change that leaves the forward's kernels as they
are leaves the sources as they were measured."""
import json
import os

import pytest

import bench


def workloads_profiled():
    with open(bench.PROFILED_TRAFFIC) as f:
        return sorted(json.load(f))


@pytest.mark.parametrize("workload", workloads_profiled())
def test_profiled_counters_are_there(workload):
    rec = bench.profiled_counters(workload)
    assert rec.get("attention_bytes_per_launch", 0) > 0 and rec.get("combine_bytes_per_launch", 0) > 0
    assert rec.get("attention_mfma_busy_pct", 0) > 0
    assert os.path.exists(os.path.join(bench.ROOT, rec["source"]))
