"""The bench's measured traffic of the weight stream belongs to the sources that were captured."""
import bench


def test_traffic_is_reported_for_the_captured_sources():
    """Helpers of other kernels belong in headers of their own: a change of these three makes the figure null."""
    assert bench.gemv_traffic_bytes() == bench.GEMV_TRAFFIC["bytes"]
