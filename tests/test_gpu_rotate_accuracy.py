"""Norm and rotation of queries and keys on inputs where sums and ranges are at stake, against the formula in float64."""
import numpy as np
import pytest
import torch

from paper_2203_15952_amd import binding as B
from test_gpu_rotate import BWD_STEPS, F, FWD_STEPS, U, Plain, dev, host
from test_gpu_rotate import test_backward as check_backward
from test_gpu_rotate import test_forward as check_forward

pytestmark = pytest.mark.gpu


# whole 16-byte pieces whose rotated halves are none: heads of each width that has a kernel of its own
PIECES_APART = [(3, 11, 4, 2, 20, 20, 0, True, True, [0, 5, 100000]), (2, 33, 3, 3, 28, 12, 0, True, True, None), (2, 17, 8, 2, 64, 62, 0, True, True, None),
                (2, 19, 6, 2, 100, 100, 0, True, True, [7, 0]), (1, 70, 2, 1, 128, 124, 0, False, False, None)]


@pytest.mark.parametrize("case", PIECES_APART)
def test_pieces_whose_halves_are_none(case):
    check_forward(case)
    check_backward(case)


@pytest.mark.parametrize("dh", [8, 7])
def test_gains_of_many_rows(dh):
    """The first rows of every lane a term of 1, all others 2^-25 and a little less, which a float32 sum would lose one by one: of a term
    16 steps, eight terms of a lane, its groups' sums, the workgroup's word and the result."""
    M, heads = 1 << 22, 1            # 256 rows to a lane: 1024 workgroups take 16384 rows at a time
    print("gains", M, dh, flush=True)
    x = torch.ones((M, 3 * dh), device="cuda")
    dy = torch.full((M, 3 * dh), 0.9 * 2.0 ** -25, device="cuda")
    dy[:16384] = 1.0
    _, dq, dk = B.aqt_qk_norm_rotate_bwd(x, dy, 1, M, B.QkNormRotate(heads, heads, dh, rot=0), dqkv=dy.clone())
    want = (dy[:, 0].double().sum() / (1.0 + 1e-6) ** 0.5).item()
    for d in (dq, dk):
        assert (d.double() / want - 1).abs().max().item() <= (16 + 8 + 4 + 1 + 1) * U


@pytest.mark.parametrize("dh,rot,pairing,shift", [(64, 64, 0, 0), (36, 36, 1, 0), (20, 20, 0, 0), (101, 100, 0, 0), (128, 64, 0, 0), (64, 62, 1, 1)])
@pytest.mark.parametrize("eps", [0.0, 1e-35])
def test_heads_of_all_sizes(dh, rot, pairing, shift, eps):
    """Columns whose squares float32 does not hold, one head of each size in a row, with next to no epsilon or none."""
    print("sizes", dh, rot, pairing, shift, eps, flush=True)
    sizes = np.array([1.0, 1e-20, 3e-38, 1e20, 1e-10, 1e38, 1e-30, 1e15, 1, 1e-25], F)      # eight queries, one key, its value
    rng = np.random.default_rng(dh)
    B_, T, heads, kv = 2, 9, 8, 1
    x, dy = (rng.uniform(-1, 1, (B_ * T, 10, dh)).astype(F) * sizes[:, None] for _ in range(2))   # dx is about 1 then
    x, dy = x.reshape(B_ * T, -1), dy.reshape(B_ * T, -1)
    gq = (1 + 0.3 * rng.standard_normal(dh)).astype(F)
    spec = B.QkNormRotate(heads, kv, dh, rot=rot, pairing=pairing, eps=eps, gamma_q=dev(gq))
    plain = Plain(B_, T, heads, kv, dh, rot, pairing, True, gq, None, 10000.0, None, eps=float(F(eps)))

    def placed(a):     # off the 16-byte boundaries with shift
        room = torch.zeros(a.size + 4, device="cuda")
        view = room[shift:shift + a.size].view(a.shape)
        view.copy_(dev(a))
        return view
    out = host(B.aqt_qk_norm_rotate_fwd(placed(x), B_, T, spec))
    ref, mag = plain.forward(x)
    assert (np.abs(out - ref) <= FWD_STEPS * U * mag + 1e-30).all()
    dx = host(B.aqt_qk_norm_rotate_bwd(placed(x), placed(dy), B_, T, spec, want_gamma=False)[0])
    ref, mag, _, _ = plain.backward(x, dy)
    q = x.reshape(B_ * T, 10, dh)[:, :9].astype(np.float64)
    r = np.concatenate([1 / np.sqrt((q * q).mean(-1) + float(F(eps))), np.zeros((B_ * T, 1))], 1)     # a step of the smallest gradients, times 1 / rms
    slack = np.repeat(2.0 ** -149 * dh * r, dh, axis=1)
    # The mean of g x^ over the head of 1e38: dh terms of 1e38 / 2 and x^ of about 1 each add up to 3.2e39 and more in magnitudes for dh
    # of 64, 1e39 for 20, where float32 ends at 3.4e38.  A float32 sum cannot be asked for it; the heads beside it can.
    fits = np.repeat(np.abs(dy.reshape(B_ * T, 10, dh)).sum(2, dtype=np.float64) < 3.4e38, dh, axis=1)
    assert fits.reshape(B_ * T, 10, dh)[:, np.arange(10) != 5].all()
    assert (np.abs(dx - ref) <= BWD_STEPS * U * mag + slack + 1e-30)[fits].all()


def test_gains_change_in_place_only():
    """An optimizer's step changes them under the spec; another tensor in their place would leave it with freed memory."""
    g = torch.ones(8, device="cuda")
    spec, x = B.QkNormRotate(1, 1, 8, rot=0, gamma_q=g), torch.ones((1, 24), device="cuda")
    before = B.aqt_qk_norm_rotate_fwd(x, 1, 1, spec)
    with pytest.raises(AttributeError):
        spec.gamma_q = torch.ones(8, device="cuda")
    g.mul_(2.0)
    after = B.aqt_qk_norm_rotate_fwd(x, 1, 1, spec)
    assert torch.equal(after[:, :8], 2 * before[:, :8]) and torch.equal(after[:, 8:], before[:, 8:])
