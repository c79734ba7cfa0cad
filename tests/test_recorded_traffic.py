"""The DRAM traffic that bench.py reports belongs to the kernels as they are."""
import bench


def test_the_recorded_captures_are_of_these_sources():
    for workload in ("c4_ffn", "c3_conv1x1"):
        assert bench.recorded_traffic(workload), workload
