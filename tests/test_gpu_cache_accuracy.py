"""The attention over the quantized cache on what a cache of real streams holds: frames whose values, keys and queries are of very
different sizes, in every form of the kernels, against float64 on what the codes stand for."""
import numpy as np
import pytest

from paper_2203_15952_amd import binding as B
from test_gpu_cache import F, U, dev, host, make, say

pytestmark = pytest.mark.gpu

# streams, capacity, heads, kv_heads, dh, bits, frames, new ones of them: a few rows, tiles of sixteen, both from several splits, and a
# wavefront to every tile
FORMS = [(1, 256, 1, 1, 64, 8, 200, 1), (2, 256, 4, 2, 36, 4, 200, 2), (1, 256, 8, 2, 128, 8, 200, 1), (2, 192, 2, 2, 20, 8, 180, 17),
         (1, 256, 12, 1, 128, 4, 200, 2), (1, 4096, 2, 2, 64, 8, 4000, 2), (1, 4096, 3, 1, 80, 4, 4000, 20), (33, 128, 8, 8, 64, 8, 128, 128),
         (16, 128, 8, 4, 100, 4, 120, 120)]


def expected(ref, rows, T, left, right, wide=False):
    """ctx of the last T frames in float64, and what an output may be off by.  A score: the query's digits are off by half a unit of
    its largest column over 2^23, so by U max|q| sum|k| / sqrt(dh), and eight roundings of it and of its distance from the largest
    (a frame 110 below it weighs nothing, and its roundings neither); twice that in the quotient.  A weight, probability times scale: an
    integer of which the largest of a tile is 2^21 at least, so half a unit is 4 U of it, for each of 64 frames; four roundings for
    every tile, the sum of weights sixteen.  Relative to the sum of the weights times the frames' largest values.
    wide: rows in which a column stands out far; their digits go on for 23 bits, and what is left is the rounding of the sums, U of the
    products' magnitudes."""
    x = rows.reshape(ref.n, T, -1, ref.dh)
    out, tol = np.zeros((ref.n, T, ref.heads, ref.dh)), np.zeros((ref.n, T, ref.heads, 1))
    g = ref.heads // ref.kv
    for b in range(ref.n):
        end = ref.end(b)
        k, v = (np.repeat(a[b].astype(np.float64), g, axis=1).transpose(1, 0, 2) for a in (ref.k, ref.v))    # [heads, frames, dh]
        q = x[b, :, :ref.heads].astype(np.float64).transpose(1, 0, 2)
        f, j = end - T + np.arange(T), np.arange(end)
        seen = (j[None] >= f[:, None] - left if left >= 0 else np.ones((T, end), bool)) & (j[None] <= f[:, None] + right if right >= 0 else True)
        s = q @ k.transpose(0, 2, 1) / np.sqrt(ref.dh)
        score = np.where(seen[None], s, -np.inf)
        p = np.exp(score - score.max(2, keepdims=True))
        p /= p.sum(2, keepdims=True)
        out[b] = (p @ v).transpose(1, 0, 2)
        mag = (p * np.abs(v).max(2)[:, None]).sum(2)
        reach = np.abs(q).max(2) * (np.where(seen[None], np.abs(k).sum(2)[:, None], 0).max(2)) / np.sqrt(ref.dh)
        if wide:
            reach = np.where(seen[None], np.abs(q) @ np.abs(k).transpose(0, 2, 1), 0).max(2) / np.sqrt(ref.dh) + reach * 2.0 ** -23
        spread = np.minimum(score.max(2) - np.where(seen[None], s, np.inf).min(2), 110.0)
        e = U * reach + 8 * U * np.where(seen[None], np.abs(s), 0).max(2) + U * (spread + 8)
        tol[b, :, :, 0] = ((2 * e + (256 + 20 * (end / 64 + 2) + 30) * U) * mag).T
    return out.reshape(ref.n * T, -1), np.broadcast_to(tol, out.shape).reshape(ref.n * T, -1)


def run(form, change, left=-1, right=0):
    """The form's frames, after change(queries, keys, values) in place ([streams, frames, heads, dh] each), through the cache."""
    streams, capacity, heads, kv, dh, bits, n, T = form
    rng = np.random.default_rng(n + T + dh)
    rows = (2 * rng.uniform(-1, 1, (streams, n, heads + 2 * kv, dh))).astype(F)
    change(rows[:, :, :heads], rows[:, :, heads:heads + kv], rows[:, :, heads + kv:])
    cache, ref = make(streams, capacity, heads, kv, dh, bits)
    if n > T:
        old = np.ascontiguousarray(rows[:, :n - T]).reshape(-1, ref.cols)
        B.aqt_cache_append(dev(old), cache, n - T, heads)
        ref.append(old, n - T)
        cache.advance(n - T)
    new = np.ascontiguousarray(rows[:, n - T:]).reshape(-1, ref.cols)
    B.aqt_cache_append(dev(new), cache, T, heads)
    ref.append(new, T)
    return host(B.aqt_attention_cached_fwd(dev(new), cache, T, heads, left=left, right=right)[0]), ref, new


def compare(form, change, left=-1, right=0, wide=False):
    got, ref, new = run(form, change, left, right)
    want, tol = expected(ref, new, form[-1], left, right, wide)
    err = np.abs(got - want)
    say("  worst", (err / (tol + 1e-30)).max(), "of its tolerance")
    assert (err <= tol + 1e-30).all()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("lift,size", [(10, 0.03), (14, 0.0), (20, 0.0)])
def test_most_of_the_weight_and_next_to_no_value(form, lift, size):
    """A first frame that draws `lift` more than the others, as attention sinks do."""
    say("sink", form, lift, size)

    def change(q, k, v):
        q[..., 0], k[..., 0], k[:, 0] = 3.0, 0.0, 0.0
        k[:, 0, :, 0] = lift * np.sqrt(form[4]) / 3
        v[:, 0] *= F(size)
    compare(form, change)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("size", [1e3, 1e5, 1e7])
def test_large_values_where_no_weight_is(form, size):
    """The call's last frame, which the rows in front of it do not see, and one that nobody listens to."""
    say("large", form, size)

    def change(q, k, v):
        q[..., 0], k[..., 0] = 4.0, 0.0
        k[:, -5, :, 0] = -30 * np.sqrt(form[4])
        v[:, -1] *= F(size)
        v[:, -5] *= F(size)
    compare(form, change)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window", [(-1, -1), (50, 2)])
def test_values_of_all_sizes(form, window):
    say("sizes", form, window)
    rng = np.random.default_rng(form[-1])

    def change(q, k, v):
        q *= F(3)
        v *= np.exp2(rng.uniform(-20, 0, v.shape[:2])).astype(F)[:, :, None, None]
    compare(form, change, *window)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("in_key", [False, True])
def test_numbers_that_are_none(form, bad, in_key):
    """In one column of one frame's key or value: the head reads back as NaN, and the rows that see the frame are NaN in every column;
    the others come out as if it were not there.  The frame: one from the middle of the call's, which half of its rows see."""
    streams, capacity, heads, kv, dh, bits, n, T = form
    say("none", form, bad, in_key)
    rng = np.random.default_rng(n + T + dh)
    rows = rng.standard_normal((streams, n, heads + 2 * kv, dh)).astype(F)
    at, head = n - 1 - T // 2, kv - 1
    clean = rows.copy()
    rows[-1, at, heads + head + (0 if in_key else kv), dh // 2] = bad
    cache, ref = make(streams, capacity, heads, kv, dh, bits)
    for lo, hi in ((0, n - T), (n - T, n)):
        if hi > lo:
            status = B.new_status()
            new = dev(np.ascontiguousarray(rows[:, lo:hi]).reshape(-1, ref.cols))
            B.aqt_cache_append(new, cache, hi - lo, heads, dev_status=status)
            assert host(status)[0] == (B.AQT_ERR_NONFINITE if lo <= at < hi else 0)
            ref.append(np.ascontiguousarray(clean[:, lo:hi]).reshape(-1, ref.cols), hi - lo)
            if hi < n:
                cache.advance(hi - lo)
    got, m = B.aqt_attention_cached_fwd(new, cache, T, heads, left=T, right=0, want_absmax=True)
    want, tol = expected(ref, clean[:, n - T:].reshape(-1, ref.cols), T, T, 0)
    got, want, tol = (a.reshape(streams, T, kv, heads // kv, dh) for a in (host(got), want, tol))
    sees = np.arange(n - T, n) >= at
    assert sees.any() and np.isnan(got[-1, sees, head]).all() and np.isnan(float(m))
    keep = np.ones(got.shape, bool)
    keep[-1, sees, head] = False
    assert (np.abs(got - want) <= tol + 1e-30)[keep].all()
    keys, values = (host(t).reshape(streams, n, kv, dh) for t in B.aqt_cache_read(cache, n, pending=T))
    hit = np.zeros(keys.shape, bool)
    hit[-1, at, head] = True
    np.testing.assert_array_equal(np.isnan(keys), hit & in_key)
    np.testing.assert_array_equal(np.isnan(values), hit & (not in_key))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("qs,ks", [(1e-30, 1e30), (1e30, 1e-30), (1e-28, 1e28)])
def test_scores_of_ordinary_size_from_small_and_large_factors(form, qs, ks):
    say("factors", form, qs, ks)

    def change(q, k, v):
        q *= F(qs)
        k *= F(ks)
    compare(form, change)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("ratio,many", [(300.0, 1), (1e4, 6), (1e6, 1)])
def test_query_columns_that_stand_out(form, ratio, many):
    """... and meet keys of zero: the other columns' scores are those of float32 sums."""
    say("standing out", form, ratio, many)

    def change(q, k, v):
        q[..., 3:3 + many], k[..., 3:3 + many] = 2 * ratio, 0.0
    compare(form, change, wide=True)


@pytest.mark.parametrize("form", [f for f in FORMS if f[-1] > 1])
def test_neighbours_of_a_row_that_stands_out(form):
    say("neighbours", form)
    T, heads, dh = form[-1], form[2], form[4]

    def with_one(q, k, v):
        q[:, -1, 0, 2] = 1e5
    rows = [run(form, change)[0].reshape(-1, T, heads, dh) for change in (lambda q, k, v: None, with_one)]
    np.testing.assert_array_equal(rows[0][:, :-1], rows[1][:, :-1])
    np.testing.assert_array_equal(rows[0][:, -1, 1:], rows[1][:, -1, 1:])
