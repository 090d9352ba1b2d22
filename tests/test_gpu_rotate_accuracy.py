"""Norm and rotation of queries and keys on inputs where sums and ranges are at stake, against the formula in float64."""
import pytest
import torch

from paper_2203_15952_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


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
