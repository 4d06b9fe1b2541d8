"""CPU-only check of the time of an iteration that the benchmark works out from whole builds."""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def test_time_of_an_iteration():
    import bench
    assert bench.lloyd_iteration_ms([14.0, 13.5, 13.75], [18.5, 18.75, 19.0]) == 1.25
    assert bench.lloyd_iteration_ms([74.0, 13.5, 13.75], [18.5, 90.0, 19.0]) == 1.25          # a stall in a build
    for two, six in (([13.5], [13.5]), ([74.0], [18.5])):                                      # none of four iterations shows: no time, rather than one below zero
        assert bench.lloyd_iteration_ms(two, six) is None
