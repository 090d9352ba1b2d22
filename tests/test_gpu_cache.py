"""The quantized cache of keys and values (codes and scales against the oracle's quantizer, bit for bit) and the attention over it
(against float64 on what those codes stand for), single calls, streams that go round their rings, and the whole chain."""
import numpy as np
import pytest
import torch

import oracle
from paper_2203_15952_amd import binding as B

pytestmark = pytest.mark.gpu
F = np.float32
U = 2.0 ** -24


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    torch.cuda.synchronize()
    return t.cpu().numpy()


def say(*a):
    print(*a, flush=True)


class Streams:
    """What every stream's cache stands for: all its frames so far, as float32 code * scale, [frames, kv_heads, dh]."""

    def __init__(self, streams, capacity, heads, kv, dh, bits):
        self.n, self.capacity, self.heads, self.kv, self.dh, self.bits = streams, capacity, heads, kv, dh, bits
        self.cols = (heads + 2 * kv) * dh
        self.k = [np.zeros((0, kv, dh), F) for _ in range(streams)]
        self.v = [np.zeros((0, kv, dh), F) for _ in range(streams)]
        self.base = np.zeros(streams, np.int64)     # frames before those kept here

    def counts(self, T, count):
        return [T if count is None else min(max(int(c), 0), T) for c in (count if count is not None else [T] * self.n)]

    def append(self, qkv, T, count=None):
        rows = qkv.reshape(self.n, T, self.heads + 2 * self.kv, self.dh)
        for b, n in enumerate(self.counts(T, count)):
            for name, h0 in (("k", self.heads), ("v", self.heads + self.kv)):
                x = np.ascontiguousarray(rows[b, :n, h0:h0 + self.kv]).reshape(-1, self.dh)
                if n:
                    q, s = oracle.quantize(x, self.bits, B.AQT_AXIS_COLS)
                    x = q.astype(F) * s[:, None]
                getattr(self, name)[b] = np.concatenate([getattr(self, name)[b], x.reshape(n, self.kv, self.dh)])

    def end(self, b):
        return int(self.base[b]) + len(self.k[b])

    def frames(self, which, b, first, n):
        out = np.zeros((n, self.kv, self.dh), F)
        x, end = getattr(self, which)[b], self.end(b)
        for i in range(n):
            p = first + i
            if max(int(self.base[b]), end - self.capacity, 0) <= p < end:
                out[i] = x[p - int(self.base[b])]
        return out

    def attention(self, qkv, T, length, count, left, right, ctx):
        """(ctx in float64, tolerance): see `tolerance` below for its terms."""
        rows = qkv.reshape(self.n, T, -1, self.dh)
        out, tol = ctx.astype(np.float64).reshape(self.n, T, self.heads, self.dh), np.zeros((self.n, T, self.heads, 1))
        g = self.heads // self.kv
        for b, n in enumerate(self.counts(T, count)):
            end, base = self.end(b), int(self.base[b])
            oldest = max(0, end - self.capacity)
            for t in range(n):
                f = int(length[b]) + t
                lo = oldest if left < 0 else max(oldest, f - left)
                hi = end - 1 if right < 0 else min(end - 1, f + right)
                if hi < lo:
                    out[b, t] = 0.0
                    continue
                k, v = (np.repeat(a[b][lo - base:hi + 1 - base].astype(np.float64), g, axis=1) for a in (self.k, self.v))
                q = rows[b, t, :self.heads].astype(np.float64)
                with np.errstate(all="ignore"):
                    s = np.einsum("hd,jhd->hj", q, k) / np.sqrt(self.dh)
                    p = np.exp(s - s.max(1, keepdims=True))
                    p /= p.sum(1, keepdims=True)
                    out[b, t] = np.einsum("hj,jhd->hd", p, v)
                    mag = (p * np.abs(v).max(2).T).sum(1)
                    tol[b, t, :, 0] = tolerance(s, np.abs(q).max(1)[:, None] * np.abs(k).sum(2).T / np.sqrt(self.dh), hi - lo + 1) * mag
        return out.reshape(self.n * T, -1), np.broadcast_to(tol, out.shape).reshape(self.n * T, -1)


def tolerance(s, reach, n):
    """Of an output, relative to sum_j p_j max|v_j|.  A score: the query's digits are off by half a unit of its largest value over
    8355584, so by U reach (reach = max|q| sum|k| / sqrt(dh)), and seven roundings of it (two of the joined sums, five products);
    the exponent takes s - max with one more.  Twice that in the quotient.  A probability's digits: half a unit of the tile's
    largest for each of its 64 frames, 64 U; every tile adds four roundings, and the sum of weights one per frame of a lane and
    tile, sixteen."""
    spread = np.abs(s - s.max(1, keepdims=True)).max(1)
    e = U * reach.max(1) + 8 * U * np.abs(s).max(1) + U * (spread + 8)
    return 2 * e + (64 + 20 * (n / 64 + 2) + 30) * U


def new_rows(rng, streams, T, cols, scale=1.0):
    return (scale * rng.standard_normal((streams * T, cols))).astype(F)


def make(streams, capacity, heads, kv, dh, bits):
    c = B.KvCache(streams, capacity, kv, dh, bits)
    c.data.fill_(255)          # NaN scales, codes of all ones: nothing that was not written may be looked at
    return c, Streams(streams, capacity, heads, kv, dh, bits)


# streams, capacity, heads, kv_heads, dh, bits
SHAPES = [(3, 64, 2, 2, 64, 8), (2, 128, 4, 4, 36, 4), (1, 192, 6, 2, 128, 4), (4, 64, 3, 1, 5, 6), (2, 128, 1, 1, 80, 8), (5, 64, 8, 2, 16, 2),
          (2, 64, 2, 1, 127, 3), (1, 64, 1, 1, 1, 5)]


@pytest.mark.parametrize("shape", SHAPES)
def test_write_and_read_back(shape):
    streams, capacity, heads, kv, dh, bits = shape
    say("cache", shape)
    rng = np.random.default_rng(sum(shape))
    cache, ref = make(*shape)
    status = B.new_status()
    for step, T in enumerate([1, 3, capacity - 2, 1, 1, capacity + 37, 2]):
        rows = new_rows(rng, streams, T, ref.cols)
        rows[0, heads * dh:] = 0.0                                  # scales of zero
        rows[-1, heads * dh:] *= 1e-38                              # ... and of next to nothing
        count = None if step % 2 == 0 else rng.integers(-1, T + 3, streams).astype(np.int32)
        cd = None if count is None else dev(count)
        B.aqt_cache_append(dev(rows), cache, T, heads, count=cd, dev_status=status)
        length = host(cache.length).copy()
        ref.append(rows, T, count)
        n = T + 6
        first = length - rng.integers(0, 9, streams)
        keys, values = (host(t).reshape(streams, n, kv, dh) for t in B.aqt_cache_read(cache, n, first=dev(first), pending=T, count=cd))
        for b in range(streams):
            np.testing.assert_array_equal(keys[b], ref.frames("k", b, int(first[b]), n))
            np.testing.assert_array_equal(values[b], ref.frames("v", b, int(first[b]), n))
        cache.advance(T, cd)
        for b in range(streams):
            assert host(cache.length)[b] == ref.end(b)
        last, none = B.aqt_cache_read(cache, 5, want_values=False)      # the last frames, as the lengths stand
        assert none is None
        for b in range(streams):
            np.testing.assert_array_equal(host(last).reshape(streams, 5, kv, dh)[b], ref.frames("k", b, ref.end(b) - 5, 5))
    assert host(status)[0] == 0


@pytest.mark.parametrize("bits", range(2, 9))
def test_every_bit_width(bits):
    cache, ref = make(2, 64, 2, 2, 40, bits)
    rows = new_rows(np.random.default_rng(bits), 2, 9, ref.cols)
    B.aqt_cache_append(dev(rows), cache, 9, 2)
    ref.append(rows, 9)
    keys, values = (host(t).reshape(2, 9, 2, 40) for t in B.aqt_cache_read(cache, 9, pending=9))
    for b in range(2):
        np.testing.assert_array_equal(keys[b], ref.frames("k", b, 0, 9))
        np.testing.assert_array_equal(values[b], ref.frames("v", b, 0, 9))


def test_untouched_bytes_unaligned_rows_and_status():
    """A call writes its own frames' bytes only; rows need no alignment; an infinity or a NaN is reported."""
    cache, ref = make(2, 64, 1, 1, 12, 8)
    rng = np.random.default_rng(3)
    rows = new_rows(rng, 2, 7, ref.cols)
    room = torch.zeros(rows.size + 1, device="cuda")
    view = room[1:].view(rows.shape)
    view.copy_(dev(rows))
    B.aqt_cache_append(view, cache, 7, 1)
    ref.append(rows, 7)
    keys, _ = B.aqt_cache_read(cache, 7, pending=7)
    np.testing.assert_array_equal(host(keys).reshape(2, 7, 1, 12)[1], ref.frames("k", 1, 0, 7))
    before = cache.data.clone()
    status = B.new_status()
    B.aqt_cache_append(view, cache, 7, 1, count=torch.tensor([0, -4], dtype=torch.int32, device="cuda"), dev_status=status)
    assert torch.equal(before, cache.data) and host(status)[0] == 0
    cache.length.fill_(3)      # frames 3 and 4: two of 64 in both streams
    B.aqt_cache_append(view[:2].contiguous(), cache, 1, 1)
    changed = host(before != cache.data).sum()
    assert 0 < changed <= 2 * 2 * (16 + 4)
    for bad in (np.inf, np.nan):
        for col in (12 + 5, 24 + 11):
            r = rows.copy()
            r[9, col] = bad
            status = B.new_status()
            B.aqt_cache_append(dev(r), cache, 7, 1, dev_status=status)
            assert host(status)[0] == B.AQT_ERR_NONFINITE
    r = rows.copy()
    r[9, 3] = np.nan           # a query: not this call's business
    status = B.new_status()
    B.aqt_cache_append(dev(r), cache, 7, 1, dev_status=status)
    assert host(status)[0] == 0


def test_lengths_far_beyond_32_bits_and_negative_ones():
    cache, ref = make(3, 64, 2, 1, 32, 8)
    far = np.array([2 ** 33 + 11, 2 ** 40 + 63, -5], np.int64)
    cache.length.copy_(dev(far))
    ref.base[:] = np.maximum(far, 0)
    rng = np.random.default_rng(8)
    rows = new_rows(rng, 3, 60, ref.cols)
    B.aqt_cache_append(dev(rows), cache, 60, 2)
    ref.append(rows, 60)
    start = ref.base.copy()
    keys, _ = B.aqt_cache_read(cache, 60, first=dev(start), pending=60)
    for b in range(3):
        np.testing.assert_array_equal(host(keys).reshape(3, 60, 1, 32)[b], ref.frames("k", b, int(start[b]), 60))
    cache.advance(60)
    assert host(cache.length).tolist() == (start + 60).tolist()
    rows = new_rows(rng, 3, 4, ref.cols)
    B.aqt_cache_append(dev(rows), cache, 4, 2)
    ref.append(rows, 4)
    ctx, _ = B.aqt_attention_cached_fwd(dev(rows), cache, 4, 2, left=20, right=2)
    want, tol = ref.attention(rows, 4, start + 60, None, 20, 2, np.zeros((12, 64)))
    np.testing.assert_array_less(np.abs(host(ctx) - want), tol + 1e-30)
    for first in (-2 ** 62, 2 ** 62):
        keys, values = B.aqt_cache_read(cache, 3, first=torch.full((3,), first, dtype=torch.int64, device="cuda"), pending=4)
        assert not host(keys).any() and not host(values).any()


ATTEND = [
    # shape, steps of new frames, (left, right), scale of the queries
    ((1, 64, 1, 1, 64, 8), [1], (-1, 0), 1.0),
    ((2, 128, 8, 8, 64, 8), [40, 1, 1], (23, 0), 2.0),
    ((3, 192, 4, 4, 36, 4), [100, 17, 150], (60, 3), 2.0),
    ((1, 4096, 8, 2, 128, 4), [4000, 1, 95, 4], (-1, 0), 2.0),
    ((2, 1024, 2, 1, 64, 8), [1000, 100], (-1, -1), 3.0),
    ((2, 64, 32, 2, 16, 4), [5, 61, 3], (0, 0), 1.0),
    ((1, 512, 3, 3, 101, 8), [300, 33], (-1, 0), 2.0),
    ((5, 64, 2, 1, 7, 6), [3, 62, 1, 70], (5, 1), 1.0),
    ((40, 256, 8, 8, 64, 8), [200, 1], (-1, 0), 2.0),
    ((1, 8192, 1, 1, 64, 8), [8192, 3], (-1, 0), 4.0),
    ((2, 256, 24, 1, 80, 3), [130, 9], (-1, 0), 2.0),
]


@pytest.mark.parametrize("shape,steps,window,scale", ATTEND)
@pytest.mark.parametrize("ragged", [False, True])
def test_attention_over_the_cache(shape, steps, window, scale, ragged):
    streams, capacity, heads, kv, dh, bits = shape
    say("attend", shape, steps, window, ragged)
    rng = np.random.default_rng(sum(shape) + len(steps))
    cache, ref = make(*shape)
    for step, T in enumerate(steps):
        rows = new_rows(rng, streams, T, ref.cols)
        rows[:, :heads * dh] *= scale
        count = rng.integers(0, T + 1, streams).astype(np.int32) if ragged else None
        if ragged and streams == 1:
            count[:] = max(1, T - 1)
        cd = None if count is None else dev(count)
        rd = dev(rows)
        B.aqt_cache_append(rd, cache, T, heads, count=cd)
        length = host(cache.length).copy()
        ref.append(rows, T, count)
        if T <= 256:
            ctx = torch.full((streams * T, heads * dh), 7.0, device="cuda")
            _, m = B.aqt_attention_cached_fwd(rd, cache, T, heads, left=window[0], right=window[1], count=cd, ctx=ctx, want_absmax=True)
            got = host(ctx).copy()
            want, tol = ref.attention(rows, T, length, count, *window, np.full((streams * T, heads * dh), 7.0))
            worst = np.abs(got - want) - tol
            assert not (worst > 1e-30).any() and not np.isnan(worst).any(), (T, np.abs(got - want).max(), tol.max())
            new = (np.arange(T) < np.array(ref.counts(T, count))[:, None]).reshape(-1)
            assert (got[~new] == 7).all()
            assert host(m)[0] == (np.abs(got[new]).max() if new.any() else 0)
            B.aqt_attention_cached_fwd(rd, cache, T, heads, left=window[0], right=window[1], count=cd, ctx=ctx)
            np.testing.assert_array_equal(host(ctx), got)              # the same bits again
        cache.advance(T, cd)


@pytest.mark.parametrize("streams,capacity,heads,kv,dh,bits,T,window", [
    (40, 256, 8, 8, 36, 4, 100, (-1, 0)), (24, 192, 16, 4, 64, 8, 90, (70, 3)), (33, 128, 8, 8, 128, 8, 128, (-1, -1)),
    (35, 64, 8, 8, 20, 3, 121, (9, 0)), (16, 512, 8, 8, 64, 8, 130, (20, 0)), (41, 128, 24, 2, 100, 4, 41, (300, 2))])
def test_attention_of_many_row_tiles(streams, capacity, heads, kv, dh, bits, T, window):
    """From 1024 tiles of 16 rows on with a short window, from 2048 on with any: a wavefront has one to itself."""
    say(streams, capacity, heads, kv, dh, bits, T, window)
    group = heads // kv
    assert streams * kv * -(-T * group // 16) >= (1024 if window[0] == 20 else 2048)
    rng = np.random.default_rng(T)
    cache, ref = make(streams, capacity, heads, kv, dh, bits)
    for n in (50, T):
        rows = new_rows(rng, streams, n, ref.cols)
        count = rng.integers(-1, n + 2, streams).astype(np.int32)
        count[:3] = 0, 1, n
        cd, length = dev(count), host(cache.length)
        B.aqt_cache_append(dev(rows), cache, n, heads, count=cd)
        ref.append(rows, n, count)
        if n == T:
            start = rng.standard_normal((streams * T, heads * dh)).astype(F)
            ctx, m = B.aqt_attention_cached_fwd(dev(rows), cache, T, heads, left=window[0], right=window[1], count=cd, ctx=dev(start),
                                                want_absmax=True)
            want, tol = ref.attention(rows, T, length, count, *window, start)
            got = host(ctx)
            np.testing.assert_array_less(np.abs(got - want), tol + 1e-30)
            brought = np.concatenate([np.arange(T) < c for c in ref.counts(T, count)])
            np.testing.assert_array_equal(got[~brought], start[~brought])
            assert float(m) == np.abs(got[brought]).max()
        cache.advance(n, cd)


@pytest.mark.parametrize("T,group", [(3, 1), (24, 1), (2, 4)])
def test_a_cache_beyond_4_gib(T, group):
    """The last head's tiles lie behind byte 2^32 of the buffer, the ring's end too."""
    kv, dh, capacity = 4, 64, 1 << 23
    say("large cache", T, group)
    heads = kv * group
    cache = B.KvCache(1, capacity, kv, dh, 8)
    assert cache.data.numel() > 1 << 32
    ref = Streams(1, capacity, heads, kv, dh, 8)
    ref.base[:] = 3 * capacity - 70
    cache.length.fill_(int(ref.base[0]))
    rng = np.random.default_rng(T)
    for n in (60, T):          # across the end of the ring
        rows = new_rows(rng, 1, n, ref.cols)
        B.aqt_cache_append(dev(rows), cache, n, heads)
        ref.append(rows, n)
        if n == 60:
            cache.advance(n)
    length = host(cache.length)
    ctx, _ = B.aqt_attention_cached_fwd(dev(rows), cache, T, heads, left=40, right=0)
    want, tol = ref.attention(rows, T, length, None, 40, 0, np.zeros((T, heads * dh)))
    np.testing.assert_array_less(np.abs(host(ctx) - want), tol + 1e-30)
    keys, values = B.aqt_cache_read(cache, 50, pending=T)
    first = ref.end(0) - 50
    np.testing.assert_array_equal(host(keys).reshape(50, kv, dh), ref.frames("k", 0, first, 50))
    np.testing.assert_array_equal(host(values).reshape(50, kv, dh), ref.frames("v", 0, first, 50))


def test_rows_beyond_2_to_31_elements():
    """A million frames at once: the last ones come out of the cache, and attend, as they do in a small call.  The outputs of the two
    calls are each within tolerance() of the same value; with scores under 16 and at most 4 frames that is (226 + 134) U of max|v|."""
    T, heads, kv, dh = 1 << 20, 16, 16, 128
    say("large rows", T)
    rows = torch.randn((T, (heads + 2 * kv) * dh), device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    cache, small = B.KvCache(1, T, kv, dh), B.KvCache(1, 256, kv, dh)
    B.aqt_cache_append(rows, cache, T, heads)
    B.aqt_cache_append(rows[-200:-100], small, 100, heads)
    small.advance(100)
    B.aqt_cache_append(rows[-100:], small, 100, heads)
    for big, want in zip(B.aqt_cache_read(cache, T, pending=T), B.aqt_cache_read(small, 200, pending=100)):
        assert big.numel() >= 1 << 31 and torch.equal(big[-200:], want)
        del big
    ctx, _ = B.aqt_attention_cached_fwd(rows, cache, T, heads, left=3)
    assert ctx.numel() >= 1 << 31
    want, _ = B.aqt_attention_cached_fwd(rows[-100:], small, 100, heads, left=3)
    top = float(rows[-200:, (heads + kv) * dh:].abs().max())
    np.testing.assert_allclose(host(ctx[-100:]), host(want), rtol=0, atol=2 * 360 * U * top)


def test_rows_that_see_nothing_are_zeros():
    """More new frames than the cache holds: the first ones' windows lie before its oldest frame."""
    cache, ref = make(1, 64, 2, 1, 32, 8)
    rows = new_rows(np.random.default_rng(0), 1, 130, ref.cols)
    B.aqt_cache_append(dev(rows), cache, 130, 2)
    ref.append(rows, 130)
    ctx = torch.full((130, 64), np.nan, device="cuda")
    B.aqt_attention_cached_fwd(dev(rows), cache, 130, 2, left=10, right=0, ctx=ctx)
    got = host(ctx)
    assert not got[:66].any()                                  # frame 65 sees 55 .. 65, the oldest held is 66
    want, tol = ref.attention(rows, 130, [0], None, 10, 0, np.zeros((130, 64)))
    np.testing.assert_array_less(np.abs(got - want), tol + 1e-30)


def test_extreme_scores_and_values():
    """Scores in the thousands (one frame takes all), queries of zeros (the mean), scales next to the ends of the range."""
    heads, dh, n = 2, 64, 200
    rng = np.random.default_rng(4)
    for qs, ks, vs in ((0.0, 1.0, 1.0), (300.0, 30.0, 1.0), (1e-30, 1.0, 1.0), (1e15, 1e15, 1.0), (1.0, 1.0, 1e30), (1.0, 1.0, 1e-25), (1.0, 1e-25, 1.0)):
        cache, ref = make(1, 256, heads, heads, dh, 8)
        rows = new_rows(rng, 1, n, ref.cols)
        rows[:, :128] *= F(qs)
        rows[:, 128:256] *= F(ks)
        rows[:, 256:] *= F(vs)
        B.aqt_cache_append(dev(rows), cache, n, heads)
        ref.append(rows, n)
        ctx, _ = B.aqt_attention_cached_fwd(dev(rows), cache, n, heads, left=-1, right=0)
        want, tol = ref.attention(rows, n, [0], None, -1, 0, np.zeros((n, 128)))
        got = host(ctx)
        assert np.isfinite(got).all()
        if qs * ks < 1e20:     # beyond, the tolerance of a score is larger than the distance between scores
            np.testing.assert_array_less(np.abs(got - want), tol + 1e-30)


def test_a_nonfinite_query_is_a_nan_in_its_own_row():
    cache, ref = make(2, 64, 4, 2, 64, 8)
    rows = new_rows(np.random.default_rng(5), 2, 3, ref.cols)
    B.aqt_cache_append(dev(rows), cache, 3, 4)
    clean = host(B.aqt_attention_cached_fwd(dev(rows), cache, 3, 4)[0])
    for bad in (np.nan, np.inf, -np.inf):
        r = rows.copy()
        r[1, 70] = bad         # frame 1 of stream 0, query head 1
        got = host(B.aqt_attention_cached_fwd(dev(r), cache, 3, 4)[0])
        assert np.isnan(got[1, 64:128]).all()
        keep = np.ones_like(got, bool)
        keep[1, 64:128] = False
        np.testing.assert_array_equal(got[keep], clean[keep])


def test_on_another_stream():
    cache, ref = make(2, 128, 4, 4, 64, 8)
    rows = dev(new_rows(np.random.default_rng(6), 2, 50, ref.cols))
    B.aqt_cache_append(rows, cache, 50, 4)
    want = host(B.aqt_attention_cached_fwd(rows, cache, 50, 4)[0])
    other, _ = make(2, 128, 4, 4, 64, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.aqt_cache_append(rows, other, 50, 4)
        ctx, _ = B.aqt_attention_cached_fwd(rows, other, 50, 4)
    side.synchronize()
    np.testing.assert_array_equal(host(ctx), want)


def test_binding_refuses():
    cache = B.KvCache(2, 64, 1, 8)
    rows = torch.zeros((6, 32), device="cuda")
    for call in (lambda **k: B.aqt_cache_append(rows, cache, **k), lambda **k: B.aqt_attention_cached_fwd(rows, cache, **k)):
        with pytest.raises(TypeError):
            call(T=2, heads=2)
        with pytest.raises(TypeError):
            call(T=3, heads=3)
        with pytest.raises(TypeError):
            call(T=3, heads=2, count=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(TypeError):
        B.aqt_attention_cached_fwd(rows, cache, 3, 2, ctx=torch.zeros((6, 15), device="cuda"))
    with pytest.raises(B.AqtError) as e:
        B.aqt_attention_cached_fwd(rows, cache, 3, 2, ws=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == B.AQT_ERR_WORKSPACE
    with pytest.raises(TypeError):
        B.aqt_attention_cached_fwd(rows, cache, 3, 2, ws=torch.empty(1 << 16, dtype=torch.uint8))
    with pytest.raises(TypeError):
        B.aqt_cache_append(rows, cache, 3, 2, dev_status=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(AttributeError):
        cache.length = torch.zeros(2, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError):
        B.KvCache(2, 64, 1, 8, length=torch.zeros(3, dtype=torch.int64, device="cuda"))
    with pytest.raises(B.AqtError):
        B.KvCache(2, 65, 1, 8)


# ---- together, as they are used ----------------------------------------------------------------------------------------


class Module:
    """Self-attention of a streaming layer out of the library's calls: quantized projection, norm and rotation, cache, attention
    over it, quantized output projection (its activations' scale from the attention's own maximum)."""

    def __init__(self, rng, streams, capacity, D, heads, kv, dh, bits):
        self.heads, self.cols = heads, (heads + 2 * kv) * dh
        self.wqkv, self.bqkv = dev((rng.standard_normal((D, self.cols)) / np.sqrt(D)).astype(F)), dev((0.1 * rng.standard_normal(self.cols)).astype(F))
        self.wo, self.bo = dev((rng.standard_normal((heads * dh, D)) / np.sqrt(heads * dh)).astype(F)), dev((0.1 * rng.standard_normal(D)).astype(F))
        self.spec = B.QkNormRotate(heads, kv, dh, gamma_q=dev((1 + 0.1 * rng.standard_normal(dh)).astype(F)), gamma_k=dev((1 + 0.1 * rng.standard_normal(dh)).astype(F)))
        self.cache = B.KvCache(streams, capacity, kv, dh, bits)
        self.wq, self.s_w, _, _ = B.aqt_quantize_weights(self.wo, 8, want_kn=False)
        self.status, self.streams, self.D = B.new_status(), streams, D

    def step(self, x, T, left, count=None):
        qkv = B.aqt_dense_fwd(x, self.wqkv, 8, 8, bias=self.bqkv, dev_status=self.status)
        return self.attend(qkv, T, left, count)

    def attend(self, qkv, T, left, count=None):
        B.aqt_qk_norm_rotate_fwd(qkv, self.streams, T, self.spec, first=self.cache.length, out=qkv)
        B.aqt_cache_append(qkv, self.cache, T, self.heads, count=count, dev_status=self.status)
        ctx, m = B.aqt_attention_cached_fwd(qkv, self.cache, T, self.heads, left=left, right=0, count=count, want_absmax=True)
        self.cache.advance(T, count)
        q, s, _ = B.aqt_quantize_with_absmax(ctx, 8, m, dev_status=self.status)
        y, _ = B.aqt_dense_fwd_q(q, s, self.wq, self.s_w, self.D, 8, 8, bias=self.bo)
        return ctx, y


@pytest.mark.parametrize("kv,bits,left", [(4, 8, 65), (2, 4, -1), (4, 8, -1)])
def test_streaming_in_chunks_is_the_whole_utterance(kv, bits, left):
    """Frame by frame, in chunks, and all at once: keys are rotated by the same positions and quantized one by one, so every way
    attends over the same codes; and with a key / value head for each query head that is what aqt_attention_fwd makes of them."""
    streams, D, heads, dh, T, capacity = 3, 96, 4, 32, 150, 192
    rng = np.random.default_rng(11 + kv)
    m = Module(rng, streams, capacity, D, heads, kv, dh, bits)
    qkv = B.aqt_dense_fwd(dev(new_rows(rng, streams, T, D)), m.wqkv, 8, 8, bias=m.bqkv).view(streams, T, m.cols)
    parts = {}
    for name, cut in (("whole", [T]), ("chunks", [16] * 9 + [6]), ("frames", [64, 50] + [1] * 36)):
        m.cache.length.zero_()
        m.cache.data.fill_(255)
        out, at = [], 0
        for n in cut:
            out.append(m.attend(qkv[:, at:at + n].reshape(streams * n, m.cols).clone(), n, left)[0].view(streams, n, heads * dh))
            at += n
        parts[name] = host(torch.cat(out, 1)).astype(np.float64)
        keys, values = (host(t).reshape(streams, T, kv, dh) for t in B.aqt_cache_read(m.cache, T))
        if name == "whole":
            first_keys, first_values = keys, values
        np.testing.assert_array_equal(keys, first_keys)
        np.testing.assert_array_equal(values, first_values)
    assert host(m.status)[0] == 0
    # one attention in float64 over those codes, with the rotated queries
    rot = host(B.aqt_qk_norm_rotate_fwd(qkv.reshape(-1, m.cols).contiguous(), streams, T, m.spec))
    ref = Streams(streams, capacity, heads, kv, dh, bits)
    ref.k, ref.v = list(first_keys), list(first_values)
    want, tol = ref.attention(rot, T, np.zeros(streams, np.int64), None, left, 0, np.zeros((streams * T, heads * dh)))
    for name, got in parts.items():
        np.testing.assert_array_less(np.abs(got.reshape(want.shape) - want), tol + 1e-30, err_msg=name)
    if kv == heads:
        fused = np.concatenate([rot[:, :heads * dh], first_keys.reshape(streams * T, -1), first_values.reshape(streams * T, -1)], 1)
        ctx, _ = B.aqt_attention_fwd(dev(fused), streams, T, heads, left=left, right=0)
        # the float attention's own error (test_gpu_attention.py): 2 (2 (dh + 2) U smag + (T + 16) U) of vmag; both are below tol's mag
        reach = np.abs(fused[:, :heads * dh]).max() * np.abs(first_keys).sum(-1).max() / np.sqrt(dh)
        slack = 2 * (2 * (dh + 2) * U * reach + (T + 16) * U) * np.abs(first_values).max()
        np.testing.assert_array_less(np.abs(host(ctx) - want), slack)


def test_the_whole_module_step_by_step():
    """Projection to projection on ragged streams: the output projection's codes are the oracle's on the attention's own output."""
    streams, D, heads, kv, dh = 4, 128, 4, 2, 32
    rng = np.random.default_rng(20)
    m = Module(rng, streams, 64, D, heads, kv, dh, 8)
    for T in (20, 1, 1, 30, 40):
        count = dev(rng.integers(1, T + 1, streams).astype(np.int32))
        ctx, y = m.step(dev(new_rows(rng, streams, T, D)), T, 40, count)
        c = host(ctx)
        q, s = oracle.quantize(c, 8, B.AQT_AXIS_ALL)
        wq, sw = oracle.quantize(host(m.wo), 8, B.AQT_AXIS_ROWS)
        want = oracle.dense_fwd_q(q, s[0], wq, sw, host(m.bo))
        from parity_util import check_forward
        check_forward(host(y), dict(want, xq=q), s[0], sw, host(m.bo), 0)
    assert host(m.status)[0] == 0


def test_a_captured_step_follows_the_lengths():
    """One decoding step, captured once: its replays go on where the lengths on the device stand, with eager work between them;
    two graphs that share a workspace and run one after the other."""
    streams, D, heads, kv, dh = 2, 64, 4, 2, 32
    rng = np.random.default_rng(30)

    def steps(m, x, graphs):
        out = []
        for i in range(8):
            m.x.copy_(x[i])
            if graphs:
                graphs[i % 2].replay()
            else:
                m.body()
            out.append((host(m.ctx).copy(), host(m.y).copy(), host(m.cache.length).copy()))
            torch.zeros(1000, device="cuda").normal_().sum().item()      # the program's own work in between
        return out

    def build():
        r = np.random.default_rng(31)
        m = Module(r, streams, 64, D, heads, kv, dh, 4)
        m.x = torch.zeros((streams, D), device="cuda")
        m.qkv = torch.zeros((streams, m.cols), device="cuda")
        m.ctx, m.y = torch.zeros((streams, heads * dh), device="cuda"), torch.zeros((streams, D), device="cuda")
        m.ws = B.workspace(1 << 20)
        m.q, m.s = torch.zeros((streams, heads * dh), dtype=torch.int8, device="cuda"), torch.zeros(1, device="cuda")

        def body():
            B.aqt_dense_fwd(m.x, m.wqkv, 8, 8, bias=m.bqkv, y=m.qkv, ws=m.ws)
            B.aqt_qk_norm_rotate_fwd(m.qkv, streams, 1, m.spec, first=m.cache.length, out=m.qkv)
            B.aqt_cache_append(m.qkv, m.cache, 1, heads)
            _, mx = B.aqt_attention_cached_fwd(m.qkv, m.cache, 1, heads, left=-1, right=0, ctx=m.ctx, want_absmax=True, ws=m.ws)
            m.cache.advance(1)
            B.aqt_quantize_with_absmax(m.ctx, 8, mx, q=m.q, scale=m.s)
            B.aqt_dense_fwd_q(m.q, m.s, m.wq, m.s_w, D, 8, 8, bias=m.bo, y=m.y, ws=m.ws)
        m.body = body
        history = dev(new_rows(np.random.default_rng(32), streams, 60, m.cols))
        B.aqt_cache_append(history, m.cache, 60, heads)
        m.cache.advance(60)
        return m

    x = [dev(new_rows(rng, streams, 1, D)) for _ in range(8)]
    want = steps(build(), x, None)
    m = build()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    start = m.cache.length.clone()
    with torch.cuda.stream(side):
        m.body()
    torch.cuda.current_stream().wait_stream(side)
    m.cache.length.copy_(start)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.body()
        graphs.append(g)
    got = steps(m, x, graphs)
    for (c, y, l), (cw, yw, lw) in zip(got, want):
        np.testing.assert_array_equal(l, lw)
        np.testing.assert_array_equal(c, cw)
        np.testing.assert_array_equal(y, yw)
    assert want[-1][2].tolist() == [68, 68]                    # round the ring of 64


def test_training_through_the_rotation():
    """Projection rows -> norm and rotation -> aqt_attention_fwd / _bwd -> the rotation's backward, against float64 autograd of the
    same formulas, gains included."""
    B_, T, heads, dh = 2, 70, 4, 32
    D = heads * dh
    rng = np.random.default_rng(40)
    x, dctx = rng.standard_normal((B_ * T, 3 * D)).astype(F), rng.standard_normal((B_ * T, D)).astype(F)
    gq, gk = (1 + 0.2 * rng.standard_normal(dh)).astype(F), (1 + 0.2 * rng.standard_normal(dh)).astype(F)
    spec = B.QkNormRotate(heads, heads, dh, gamma_q=dev(gq), gamma_k=dev(gk), pairing=B.AQT_ROTATE_PAIRS)
    xd = dev(x)
    rot = B.aqt_qk_norm_rotate_fwd(xd, B_, T, spec)
    lse = torch.empty((B_ * T, heads), device="cuda")
    ctx, _ = B.aqt_attention_fwd(rot, B_, T, heads, left=20, right=5, lse=lse)
    drot = B.aqt_attention_bwd(rot, ctx, dev(dctx), lse, B_, T, heads, left=20, right=5)
    dqkv, dgq, dgk = B.aqt_qk_norm_rotate_bwd(xd, drot, B_, T, spec, dqkv=drot)
    xt, gqt, gkt = (torch.from_numpy(a).double().requires_grad_() for a in (x, gq, gk))
    rows = xt.view(B_, T, 3, heads, dh)
    w = torch.outer(torch.arange(T).double(), 10000.0 ** (-2 * torch.arange(dh // 2).double() / dh))
    c, s = torch.cos(w)[:, None], torch.sin(w)[:, None]

    def turned(q, g):
        n = q / ((q * q).mean(-1, keepdim=True) + 1e-6).sqrt() * g
        a, b = n[..., 0::2], n[..., 1::2]
        return torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)

    q, k, v = turned(rows[:, :, 0], gqt).transpose(1, 2), turned(rows[:, :, 1], gkt).transpose(1, 2), rows[:, :, 2].transpose(1, 2)
    off = torch.arange(T)[None] - torch.arange(T)[:, None]
    score = (q @ k.transpose(-1, -2) / dh ** 0.5).masked_fill((off < -20) | (off > 5), -torch.inf)
    out = (torch.softmax(score, -1) @ v).transpose(1, 2).reshape(B_ * T, D)
    out.backward(torch.from_numpy(dctx).double())
    # float32 chains of at most T + 2 dh + 64 roundings, against the largest gradient (the parity rule of the gradients: 1e-4)
    for got, want in ((ctx, out.detach()), (dqkv, xt.grad), (dgq, gqt.grad), (dgk, gkt.grad)):
        want = want.numpy()
        assert np.abs(host(got) - want).max() <= 2 * (T + 2 * dh + 64) * U * np.abs(want).max()
