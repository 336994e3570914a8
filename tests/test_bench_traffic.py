"""The bench's DRAM traffic figure is reported only while the head kernel's sources are those it was captured on: a change to them
has to bring a new capture, and nothing else may touch them."""
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_traffic_figure_belongs_to_the_sources():
    sys.path.insert(0, ROOT)
    import bench
    assert bench.ncu_traffic_or_none() == bench.NCU_TRAFFIC["bytes"]
