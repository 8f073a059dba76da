"""The bench's roofline row names the bytes that a triad launch moves, from
counters taken on the present kernel sources: where those have changed since, the
summary in profiles/ is to be taken again, or the bench says null.  No GPU needed."""
import bench


def test_recorded_traffic_holds_for_the_present_sources():
    assert bench.recorded_traffic() is not None
