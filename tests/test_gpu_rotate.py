"""Queries and keys normalised per head and rotated, forward and backward, against float64."""
import numpy as np
import pytest
import torch

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


class Plain:
    """The formula in float64 on rows [M, heads + 2 kv_heads, dh]."""

    def __init__(self, B_, T, heads, kv, dh, rot, pairing, norm, gq, gk, base, first, eps=1e-6):
        self.h, self.kv, self.dh, self.norm, self.eps = heads, kv, dh, norm, eps
        p = rot // 2
        frame = (np.arange(T)[None] + (np.zeros(B_, np.int64) if first is None else first)[:, None]).reshape(-1)
        w = frame.astype(np.longdouble)[:, None] * (np.longdouble(base) ** (-2 * np.arange(p, dtype=np.longdouble) / max(rot, 1)))
        self.c, self.s = np.cos(w).astype(np.float64)[:, None], np.sin(w).astype(np.float64)[:, None]
        self.a, self.b = (np.arange(p), np.arange(p) + p) if pairing == B.AQT_ROTATE_HALVES else (2 * np.arange(p), 2 * np.arange(p) + 1)
        ones = np.ones(dh)
        g = np.stack([ones if gq is None else gq] * heads + [ones if gk is None else gk] * kv).astype(np.float64)
        self.gain = g if norm else np.ones_like(g)

    def rows(self, x):
        return x.reshape(-1, self.h + 2 * self.kv, self.dh).astype(np.float64)

    def turn(self, x, sign=1.0):
        y = x.copy()
        y[..., self.a] = x[..., self.a] * self.c - sign * x[..., self.b] * self.s
        y[..., self.b] = sign * x[..., self.a] * self.s + x[..., self.b] * self.c
        return y

    def pairs(self, x):
        """What an element's rounding errors are measured against: the magnitudes of its pair."""
        m = np.abs(x)
        y = m.copy()
        y[..., self.a] = y[..., self.b] = m[..., self.a] + m[..., self.b]
        return y

    def forward(self, x):
        x = self.rows(x)
        n = self.h + self.kv
        q = x[:, :n]
        r = 1 / np.sqrt((q * q).mean(-1, keepdims=True) + self.eps) if self.norm else np.ones_like(q[..., :1])
        y = q * r * self.gain
        out = x.copy()
        out[:, :n] = self.turn(y)
        mag = np.zeros_like(x)
        mag[:, :n] = self.pairs(y)
        return out.reshape(len(x), -1), mag.reshape(len(x), -1)

    def backward(self, x, dy):
        x, d = self.rows(x), self.rows(dy)
        n = self.h + self.kv
        q = x[:, :n]
        u, umag = self.turn(d[:, :n], -1.0), self.pairs(d[:, :n])
        dx, mag = d.copy(), np.zeros_like(d)
        if not self.norm:
            dx[:, :n], mag[:, :n] = u, umag
            return dx.reshape(len(x), -1), mag.reshape(len(x), -1), None, None
        r = 1 / np.sqrt((q * q).mean(-1, keepdims=True) + self.eps)
        xh, g, gmag = q * r, u * self.gain, umag * np.abs(self.gain)
        dx[:, :n] = r * (g - xh * (g * xh).mean(-1, keepdims=True))
        mag[:, :n] = r * (gmag + np.abs(xh) * (gmag * np.abs(xh)).mean(-1, keepdims=True))
        t, tm = (u * xh).sum(0), (umag * np.abs(xh)).sum(0)
        gains = [(t[:self.h].sum(0), tm[:self.h].sum(0)), (t[self.h:].sum(0), tm[self.h:].sum(0))]
        return dx.reshape(len(x), -1), mag.reshape(len(x), -1), gains[0], gains[1]


# Rounding steps in units of U.  The sum of squares: eight products and sums per lane and up to six levels of lanes, all positive,
# halved by the root: 7; mean, eps, root, reciprocal: 3; times r and the gain: 2; a cosine: 3 (reduced angle, polynomial); two
# products and a difference: 2.
FWD_STEPS = 18
# u: 5; x^: 11; their product, the gain, and the sum over the head: 20; the difference, r once more: 12.
BWD_STEPS = 48

CASES = [
    # B, T, heads, kv, dh, rot, pairing, norm, gains, first
    (1, 1, 1, 1, 1, 0, 0, True, True, None),
    (1, 1, 1, 1, 2, 2, 1, True, True, [5]),
    (3, 1, 8, 8, 64, 64, 0, True, True, [0, 200000, 7]),
    (2, 37, 4, 4, 36, 36, 1, True, True, None),
    (2, 37, 4, 4, 36, 36, 0, True, True, [1, 2]),              # halves of 18: no whole pieces
    (5, 13, 6, 2, 48, 16, 0, True, False, [0, 1, 2, 3, 1000000]),
    (1, 129, 12, 3, 128, 128, 0, True, True, None),
    (1, 65, 2, 1, 101, 100, 0, True, True, [3]),               # odd width
    (2, 33, 3, 3, 20, 10, 1, True, True, None),                # a piece half rotated
    (4, 50, 4, 2, 64, 62, 1, False, False, None),              # rotation only
    (4, 50, 4, 2, 64, 0, 0, True, True, None),                 # norm only
    (2, 9, 2, 2, 8, 8, 0, False, False, [2 ** 31 - 5, 2 ** 40]),
    (8, 700, 2, 1, 32, 32, 0, True, True, None),               # several rows to a wavefront
    (3, 2000, 16, 16, 4, 4, 1, True, True, None),
]


def inputs(case):
    B_, T, heads, kv, dh, rot, pairing, norm, gains, first = case
    rng = np.random.default_rng(B_ * 1000 + T + dh)
    cols = (heads + 2 * kv) * dh
    x, dy = rng.standard_normal((B_ * T, cols)).astype(F), rng.standard_normal((B_ * T, cols)).astype(F)
    gq, gk = ((1 + 0.3 * rng.standard_normal(dh)).astype(F) for _ in range(2)) if gains else (None, None)
    first = None if first is None else np.array(first, np.int64)
    spec = B.QkNormRotate(heads, kv, dh, rot=rot, base=10000.0, pairing=pairing, norm=norm, gamma_q=None if gq is None else dev(gq),
                          gamma_k=None if gk is None else dev(gk))
    return x, dy, spec, None if first is None else dev(first), Plain(B_, T, heads, kv, dh, rot, pairing, norm, gq, gk, 10000.0, first)


def angle_slack(case):
    """A frame f's angle f * turns in float64 is off by two roundings of 2^-53: 2 pi times that."""
    last = max(case[9] or [0]) + case[1]
    return 4 * np.pi * last * 2.0 ** -53


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    say("rotate fwd", case)
    x, _, spec, first, plain = inputs(case)
    B_, T, heads, kv, dh = case[:5]
    xd = dev(x)
    out = host(B.aqt_qk_norm_rotate_fwd(xd, B_, T, spec, first=first))
    ref, mag = plain.forward(x)
    np.testing.assert_array_less(np.abs(out - ref), (FWD_STEPS * U + angle_slack(case)) * mag + 1e-30)
    turned = (heads + kv) * dh
    np.testing.assert_array_equal(out[:, turned:], x[:, turned:])          # the values, bit for bit
    np.testing.assert_array_equal(host(xd), x)
    B.aqt_qk_norm_rotate_fwd(xd, B_, T, spec, first=first, out=xd)         # in place: the same bits
    np.testing.assert_array_equal(host(xd), out)


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    say("rotate bwd", case)
    x, dy, spec, first, plain = inputs(case)
    B_, T, heads, kv, dh = case[:5]
    dyd = dev(dy)
    dqkv, dgq, dgk = B.aqt_qk_norm_rotate_bwd(dev(x), dyd, B_, T, spec, first=first)
    ref, mag, gq, gk = plain.backward(x, dy)
    got = host(dqkv)
    np.testing.assert_array_less(np.abs(got - ref), (BWD_STEPS * U + 2 * angle_slack(case)) * mag + 1e-30)
    np.testing.assert_array_equal(got[:, (heads + kv) * dh:], dy[:, (heads + kv) * dh:])
    if spec.norm:
        # per term 16 steps; a lane adds the heads of its rows one after the other, then lanes, wavefronts, and float64
        chain = -(-B_ * T // 4096) * (heads + kv) + 16 + 16
        for d, (r, m) in ((dgq, gq), (dgk, gk)):
            np.testing.assert_array_less(np.abs(host(d) - r), (chain * U + angle_slack(case)) * m + 1e-30)
    else:
        assert dgq is None and dgk is None
    again, dgq2, dgk2 = B.aqt_qk_norm_rotate_bwd(dev(x), dyd, B_, T, spec, first=first, dqkv=dyd)   # in place, the same bits
    assert again is dyd
    np.testing.assert_array_equal(host(dyd), got)
    if spec.norm:
        np.testing.assert_array_equal(host(dgq2), host(dgq))
        np.testing.assert_array_equal(host(dgk2), host(dgk))


@pytest.mark.parametrize("case", [c for c in CASES if c[0] * c[1] < 200])
def test_gradient_against_differences(case):
    """The gradient of sum(w * out) along a random direction, against central differences of the float64 formula."""
    x, w, spec, first, plain = inputs(case)
    B_, T, heads, kv, dh = case[:5]
    v = np.random.default_rng(5).standard_normal(x.shape)
    dqkv = host(B.aqt_qk_norm_rotate_bwd(dev(x), dev(w), B_, T, spec, first=first)[0]).astype(np.float64)
    h = 1e-6
    diff = ((plain.forward(x + h * v)[0] - plain.forward(x - h * v)[0]) * w).sum() / (2 * h)
    mag = np.abs(plain.backward(x, w)[1] * v).sum() + np.abs(w * v).sum()
    # rounding of the differences: 2^-52 / h of the sum of magnitudes; their third derivative: h^2 (rows of one column have curvature 1 / |x|^3)
    assert abs((dqkv * v).sum() - diff) <= (BWD_STEPS * U + 2.0 ** -50 / h + 1e-7) * mag


def test_unaligned_tensors_and_given_turns():
    rng = np.random.default_rng(1)
    heads, kv, dh, B_, T = 4, 2, 32, 2, 19
    cols = (heads + 2 * kv) * dh
    x = rng.standard_normal((B_ * T, cols)).astype(F)
    aligned = dev(x)
    spec = B.QkNormRotate(heads, kv, dh, rot=16)
    want = host(B.aqt_qk_norm_rotate_fwd(aligned, B_, T, spec))
    room = torch.zeros(x.size + 5, device="cuda")
    view = room[1:1 + x.size].view(B_ * T, cols)
    view.copy_(aligned)
    out = torch.full((x.size + 5,), 7.0, device="cuda")
    B.aqt_qk_norm_rotate_fwd(view, B_, T, spec, out=out[3:3 + x.size].view(B_ * T, cols))
    got = host(out)
    # the other kernel adds up the squares of a head in another order
    np.testing.assert_allclose(got[3:3 + x.size].reshape(want.shape), want, rtol=0, atol=2 * FWD_STEPS * U * 2 * np.abs(want).max())
    assert (got[:3] == 7).all() and (got[3 + x.size:] == 7).all()
    given = B.QkNormRotate(heads, kv, dh, rot=16, turns=spec.turns.clone())
    np.testing.assert_array_equal(host(B.aqt_qk_norm_rotate_fwd(aligned, B_, T, given)), want)
    np.testing.assert_allclose(host(spec.turns), 10000.0 ** (-np.arange(8) / 8) / (2 * np.pi), rtol=1e-14)


def test_more_than_2_to_30_rows():
    """Rows and bytes that do not count in 32 bits: the last utterance and one in the middle come out as they do by themselves."""
    B_, T, spec = 1025, 1 << 20, B.QkNormRotate(1, 1, 2)
    gen = torch.Generator(device="cuda").manual_seed(0)
    say("many rows", B_, T)
    x = torch.randn((B_ * T, 6), device="cuda", generator=gen)
    dy = torch.randn((B_ * T, 6), device="cuda", generator=gen)
    first = torch.arange(B_, dtype=torch.int64, device="cuda") * 1000
    some = [(b, slice(b * T, (b + 1) * T)) for b in (513, B_ - 1)]
    alone = [(B.aqt_qk_norm_rotate_fwd(x[at], 1, T, spec, first=first[b:b + 1]),
              B.aqt_qk_norm_rotate_bwd(x[at], dy[at], 1, T, spec, first=first[b:b + 1], want_gamma=False)[0]) for b, at in some]
    B.aqt_qk_norm_rotate_bwd(x, dy, B_, T, spec, first=first, dqkv=dy, want_gamma=False)
    B.aqt_qk_norm_rotate_fwd(x, B_, T, spec, first=first, out=x)
    for (b, at), (y, dx) in zip(some, alone):
        assert torch.equal(x[at], y) and torch.equal(dy[at], dx)


def test_special_values_stay_in_their_head():
    """A NaN, an infinity and a head of zeros: what the formula gives there, and nothing in the heads beside them."""
    heads, kv, dh = 4, 4, 64
    rng = np.random.default_rng(2)
    x = rng.standard_normal((6, 3 * 4 * 64)).astype(F)
    clean = host(B.aqt_qk_norm_rotate_fwd(dev(x), 1, 6, B.QkNormRotate(heads, kv, dh)))
    y = x.copy()
    y[1, 5], y[2, 64 + 3], y[3, 4 * 64:5 * 64] = np.nan, np.inf, 0.0
    y[4, 2 * 4 * 64 + 1] = -np.inf                                   # a value: passes as it is
    got = host(B.aqt_qk_norm_rotate_fwd(dev(y), 1, 6, B.QkNormRotate(heads, kv, dh)))
    assert np.isnan(got[1, :64]).all() and np.isnan(got[2, 64:128]).any() and (got[3, 4 * 64:5 * 64] == 0).all()
    assert got[4, 2 * 4 * 64 + 1] == -np.inf
    keep = np.ones_like(x, bool)
    keep[1, :64] = keep[2, 64:128] = keep[3, 256:320] = keep[4, 513] = False
    np.testing.assert_array_equal(got[keep], clean[keep])
    # without norm an infinity behind the rotated columns stays where it is
    z = x.copy()
    z[0, 11] = np.inf
    for pairing in (0, 1):
        o = host(B.aqt_qk_norm_rotate_fwd(dev(z), 1, 6, B.QkNormRotate(heads, kv, dh, rot=10, norm=False, pairing=pairing)))
        assert o[0, 11] == np.inf and np.isfinite(np.delete(o, 11, axis=1)).all()


def test_binding_refuses():
    spec = B.QkNormRotate(2, 1, 8)
    x = torch.zeros((6, 32), device="cuda")
    for bad in (x[:5], x.double(), x.t().contiguous().t(), torch.zeros((6, 33), device="cuda")):
        with pytest.raises(TypeError):
            B.aqt_qk_norm_rotate_fwd(bad, 2, 3, spec)
    with pytest.raises(TypeError):
        B.aqt_qk_norm_rotate_fwd(x, 2, 3, spec, first=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        B.aqt_qk_norm_rotate_fwd(x, 2, 3, spec, out=torch.zeros((6, 31), device="cuda"))
    with pytest.raises(TypeError):
        B.QkNormRotate(2, 1, 8, gamma_q=torch.ones(7, device="cuda"))
    with pytest.raises(ValueError):
        B.aqt_qk_norm_rotate_fwd(torch.zeros((6, 32)), 2, 3, spec)
    with pytest.raises(B.AqtError):
        B.QkNormRotate(2, 1, 8, rot=7)
    with pytest.raises(B.AqtError):
        B.aqt_qk_norm_rotate_fwd(x, 2, 3, B.QkNormRotate(2, 1, 8, pairing=3))
    for ws in (torch.empty(1 << 24, dtype=torch.uint8), torch.empty(1 << 22, device="cuda")):
        with pytest.raises(TypeError):
            B.aqt_qk_norm_rotate_bwd(x, x.clone(), 2, 3, spec, ws=ws)
    with pytest.raises(ValueError):
        B.QkNormRotate(2, 1, 8, device="cpu")
    spec.device = 1                                                  # gains and turns of another device's
    with pytest.raises(ValueError):
        B.aqt_qk_norm_rotate_fwd(x, 2, 3, spec)
    with pytest.raises(ValueError):
        B.aqt_qk_norm_rotate_bwd(x, x.clone(), 2, 3, spec)
