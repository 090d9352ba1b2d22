"""The library's version moves with its entry points, and the benchmark's traffic table names the versions whose kernels it was measured on."""
import bench
from paper_2203_15952_amd import binding as B


def test_version_counts_the_entry_points_around_positions_and_the_cache():
    assert B.lib().aqt_version() >= 203
    assert 202 in bench.PROFILED_VERSIONS
