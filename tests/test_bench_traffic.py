"""The bench line's DRAM traffic comes from counters of the streaming kernel as its sources stood when they were taken."""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def test_the_counters_are_those_of_the_sources():
    """Declarations that the streaming kernel does not use belong in other headers: any change to its own files makes the
    bench line drop its traffic figure until the counters are taken again."""
    import bench
    assert bench._traffic_still_valid()
    assert bench.NCU_TRAFFIC_BYTES_PER_ROW[3] * 256 * 5 == 2363904000       # the figure of the default line
