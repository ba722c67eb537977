"""The tiling kernel of cached tokens' weights keeps the rule of tests/test_waits.py: lanes wait alone only where one lane runs."""
import test_waits


def test_lanes_wait_alone_only_where_one_lane_runs():
    test_waits.test_lanes_wait_alone_only_where_one_lane_runs("weights_tile.cu")
