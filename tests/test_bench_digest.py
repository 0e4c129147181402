"""bench.py's DRAM traffic belongs to the kernels it was captured with."""
import bench


def test_the_captured_kernels_are_those_of_the_tree():
    """A change of the projection kernels asks for a capture of their own; until then the bench's line has no traffic."""
    assert bench.kernel_source_digest() == bench.NCU_KERNEL_SOURCE_SHA256_16
    assert bench.ncu_traffic(1.0e8) == 1.0e8 * bench.NCU_TRAFFIC_PER_WEIGHT_BYTE
