"""Group norm read in two passes where groups span slabs of channels and samples are cut into
several pixel ranges."""
import math

import pytest
import torch

from tests import test_gpu_group_norm as T

pytestmark = pytest.mark.gpu

# (K, N, P, C, G).  Channels one by one (slabs of 256), groups of 63 and 206 across their edges,
# a narrow last slab of 185 and 6; vectors (slabs of 128 in f32, 256 in 16 bits), groups of 65
# and a last slab of 8, and one group across all slabs.  12, 7, 6 and 6 pixel ranges.
SPANNING = [(1, 2, 100, 441, 7), (1, 1, 60, 1030, 5), (2, 1, 400, 520, 8), (1, 1, 400, 1024, 1)]


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", list(T.DT))
@pytest.mark.parametrize("shape", SPANNING, ids=str)
def test_groups_across_slabs(shape, dtype, act):
    T.test_forward(shape, dtype, act)
    T.test_backward(shape, dtype, act)


@pytest.mark.parametrize("shape", [(1, 32, 3408, 273, 7)] + SPANNING, ids=str)
def test_a_group_has_the_same_statistics_in_all_its_slabs(shape):
    """Channels with the same values, gamma and beta in one group get the same y and dx bit for
    bit, whichever slabs they lie in, and twice the same.  Means of 1e5 deviations: another order
    of the binary64 sums moves the variance by up to about 1e10 2^-53 = 1e-6 of itself, 20 units
    of fp32.  (Joined by 32 lanes in one slab and 64 in the other, about one group in six of
    3408 x 39 values had another rstd there; the first shape has 32 of them.)"""
    print(f"[case] {shape}", flush=True)
    S = T._S()
    K, N, P, C, G = shape
    Cg = C // G
    x, dy, gamma, beta = T._inputs(shape, "f32", 14)
    x += 1e5
    for v in (x, dy, gamma, beta):
        q = v.unflatten(-1, (G, Cg))
        q[..., -1] = q[..., 0]
    plan = T._plan(S, shape, "f32", "silu")

    def run():
        y, mean, rstd = T._forward(S, plan, x, gamma, beta)
        dx = torch.full_like(x, math.nan)
        dg, db = torch.empty((K, C), device="cuda"), torch.empty((K, C), device="cuda")
        S.saef_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, dx, dg, db)
        return y, mean, rstd, dx, dg, db
    first = run()
    for v in (first[0], first[3]):  # (y and dx; a channel's own sums follow its slab's threads)
        q = v.unflatten(-1, (G, Cg))
        assert torch.equal(q[..., -1], q[..., 0])
    for _ in range(3):
        for a, b in zip(first, run()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("shape", SPANNING, ids=str)
def test_means_far_above_the_deviation(shape):
    T.test_means_far_above_the_deviation(shape)
