"""The committed record of the fused kernel's DRAM traffic is of the sources as
they are, so that the bench line carries it: what other kernels need is kept
out of those files, and a change to them is measured again."""
import pytest

import bench
from paper_2606_00724_gb300 import synth


@pytest.mark.parametrize("workload,traffic", [("c3", 205862400), ("c4", 239130112)])
def test_record_is_of_the_current_sources(workload, traffic):
    assert bench.recorded_traffic(synth.WORKLOADS[workload]) == traffic
