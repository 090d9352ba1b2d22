"""Calls around positions and the cache that are refused before a launch (the addresses are never dereferenced)."""
import pytest

from paper_2203_15952_amd import binding as B
from test_positions_and_cache_cpu import BIG, INVALID, L, ONE, cache   # noqa: F401  (L: the fixture)


def test_reading_new_frames_by_count_names_the_call_they_came_in(L):
    """count says how many of `pending` frames a stream brought: without pending it would say nothing, and the last frames read
    would be the old ones."""
    for pending in (0, -1):
        assert L.aqt_cache_read(cache(), pending, BIG, None, 1, 2 * BIG, 3 * BIG, None) == INVALID
