"""The committed measurements that the benchmark's line quotes were taken on
the sources as they are."""
import bench


def test_decode_traffic_is_of_the_current_sources():
    assert bench.measured_traffic() is not None
