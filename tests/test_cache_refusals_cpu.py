"""Calls around positions and the cache that are refused before a launch (the addresses are never dereferenced)."""
import pytest

from paper_2203_15952_amd import binding as B
from test_positions_and_cache_cpu import BIG, INVALID, L, cache, spec   # noqa: F401  (L: the fixture)


def test_reading_new_frames_by_count_names_the_call_they_came_in(L):
    """count says how many of `pending` frames a stream brought: without pending it would say nothing, and the last frames read
    would be the old ones."""
    for pending in (0, -1):
        assert L.aqt_cache_read(cache(), pending, BIG, None, 1, 2 * BIG, 3 * BIG, None) == INVALID


AT = [k << 40 for k in range(1, 12)]     # addresses far apart


def test_append_refuses_rows_in_the_cache(L):
    c, nbytes = cache(data=AT[0], length=AT[1]), B.lib().aqt_cache_bytes(cache())
    for qkv, count, status in [(AT[0], None, None), (AT[0] + nbytes - 4, None, None), (AT[0] - 4, None, None), (AT[1], None, AT[1] + 8),
                               (AT[2], AT[0] + 64, None), (AT[2], AT[3], AT[0]), (AT[2], AT[3], AT[2] + 8), (AT[2], AT[3], AT[3])]:
        assert L.aqt_cache_append(qkv, 1, 4, c, count, None, status) == INVALID
    for length in (AT[0], AT[0] + nbytes - 8):
        assert L.aqt_cache_append(AT[2], 1, 4, cache(data=AT[0], length=length), None, None, None) == INVALID


def test_read_refuses_results_over_each_other_and_over_what_it_reads(L):
    c, nbytes = cache(data=AT[0], length=AT[1]), B.lib().aqt_cache_bytes(cache())
    n = 3
    size = 2 * n * 2 * 16 * 4
    for keys, values in [(AT[2], AT[2]), (AT[2], AT[2] + size - 4), (AT[2] + size - 4, AT[2]), (AT[0] + nbytes - 4, AT[2]), (AT[2], AT[0]),
                         (AT[1] + 8, None), (None, AT[1]), (AT[3], AT[2]), (AT[2], AT[4] + 8)]:
        assert L.aqt_cache_read(c, 1, AT[3], AT[4], n, keys, values, None) == INVALID


def test_attention_refuses_results_over_the_cache_the_workspace_and_each_other(L):
    c, nbytes = cache(data=AT[0], length=AT[1]), B.lib().aqt_cache_bytes(cache())
    need = B.lib().aqt_attention_cached_workspace_bytes(cache(), 1, 4)
    att = L.aqt_attention_cached_fwd
    good = dict(qkv=AT[2], count=AT[3], ctx=AT[4], absmax=AT[5], ws=AT[6])
    for bad in (dict(ctx=AT[0]), dict(ctx=AT[0] + nbytes - 4), dict(ctx=AT[1]), dict(ctx=AT[3]), dict(ctx=AT[6] + need - 4), dict(ctx=AT[5]),
                dict(absmax=AT[0]), dict(absmax=AT[2]), dict(absmax=AT[3] + 4), dict(absmax=AT[6]), dict(absmax=AT[4] + 4),
                dict(ws=AT[0]), dict(ws=AT[2]), dict(ws=AT[1])):
        a = good | bad
        assert att(a["qkv"], 1, 4, c, a["count"], -1, 0, a["ctx"], a["absmax"], a["ws"], need, None) == INVALID, bad


def test_advance_refuses_counts_in_the_lengths(L):
    for count in (AT[0], AT[0] + 12, AT[0] - 4):
        assert L.aqt_cache_advance(AT[0], 2, 1, count, None) == INVALID


def test_rotation_refuses_results_over_what_it_reads(L):
    s = spec(gamma_q=AT[0], gamma_k=AT[1], turns=AT[2])
    row = 6 * (4 + 2 * 2) * 16 * 4
    for out in (AT[0], AT[1] - row + 4, AT[2] + 4, AT[3]):
        assert L.aqt_qk_norm_rotate_fwd(AT[4], 2, 3, s, AT[3], out, None) == INVALID
    need = B.aqt_workspace_bytes(B.AQT_OP_QK_NORM_ROTATE_BWD, 6, 16, 1)
    good = dict(dqkv=AT[5], dgq=AT[6], dgk=AT[7], ws=AT[8])
    for bad in (dict(dqkv=AT[0]), dict(dqkv=AT[3]), dict(dgq=AT[0]), dict(dgq=AT[4]), dict(dgq=AT[9]), dict(dgk=AT[6] + 60), dict(dgk=AT[5]),
                dict(dgk=AT[2]), dict(ws=AT[4]), dict(ws=AT[9]), dict(ws=AT[5] - need + 4), dict(ws=AT[6]), dict(ws=AT[1])):
        a = good | bad
        assert L.aqt_qk_norm_rotate_bwd(AT[4], AT[9], 2, 3, s, AT[3], a["dqkv"], a["dgq"], a["dgk"], a["ws"], need, None) == INVALID, bad
    # in place the workspace must not be the gradient either
    assert L.aqt_qk_norm_rotate_bwd(AT[4], AT[9], 2, 3, s, AT[3], AT[9], AT[6], AT[7], AT[9], need, None) == INVALID
