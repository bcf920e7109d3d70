"""The gradient of group norm does not depend on the scale of the features: rstd squared leaves
fp32 long before the features do."""
import numpy as np
import pytest
import torch

from tests import operators_oracle as O
from tests import test_gpu_group_norm as T

pytestmark = pytest.mark.gpu

# one read, two reads, odd channels held, one by one with groups across slabs
SHAPES = [(2, 3, 49, 64, 8), (1, 2, 3136, 32, 4), (2, 3, 60, 30, 5), (1, 2, 100, 441, 7)]


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power,eps", [(40, 1e-5), (70, 1e-5), (100, 1e-5), (-72, 1e-44)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_features_of_any_scale(shape, power, eps, dtype, act):
    """Features times 2^power, at the bounds of the test of ordinary ones (they scale with
    rstd).  dx is about 2^-power: far from the ends of fp32."""
    print(f"[case] {shape} {power} {dtype} {act}", flush=True)
    S = T._S()
    K, N, P, C, G = shape
    eps = float(np.float32(eps))
    x, dy, gamma, beta = T._inputs(shape, dtype, 16)
    x *= 2.0 ** power  # (exact)
    hx = T._np(x)
    mean, rstd = (torch.from_numpy(v).float().cuda() for v in O.stats(hx, G, eps))
    if act == "relu":
        z = O.spread(T._np(rstd), C) * (hx - O.spread(T._np(mean), C)) * T._np(gamma)[:, None, None]
        near = np.abs(z + T._np(beta)[:, None, None]) < 1e-4
        dy.masked_fill_(torch.from_numpy(near).cuda(), 0.0)
    plan = S.GroupNorm(K, N, P, C, G, T.DT[dtype], eps=eps,
                       act={"none": S.ACT_NONE, "relu": S.ACT_RELU, "silu": S.ACT_SILU}[act])
    y, mean2, rstd2 = T._forward(S, plan, x, gamma, beta)
    want, _, _, w = O.forward(hx, T._np(gamma), T._np(beta), G, act, eps)
    rel, tiny = O.OUT[dtype]
    err = 32 * O.U * w + 1e-7 * np.abs(T._np(gamma))[:, None, None, :]
    O.assert_within(T._np(y), want, err + rel * (np.abs(want) + err) + tiny, "y")
    O.assert_within(T._np(mean2), T._np(mean), 2 * O.U * np.abs(T._np(mean))
                    + 1e-9 * 2.0 ** power, "mean")
    O.assert_within(T._np(rstd2), T._np(rstd), 2 * O.U * T._np(rstd), "rstd")
    dx = torch.full_like(x, float("nan"))
    dg, db = torch.empty((K, C), device="cuda"), torch.empty((K, C), device="cuda")
    S.saef_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, dx, dg, db)
    (wx, wg, wb), (ex, eg, eb) = O.backward(T._np(dy), hx, T._np(mean), T._np(rstd), T._np(gamma),
                                            T._np(beta), act)
    O.assert_within(T._np(dx), wx, ex + rel * (np.abs(wx) + ex) + tiny, "dx")
    O.assert_within(T._np(dg), wg, eg + O.U * np.abs(wg), "dgamma")
    O.assert_within(T._np(db), wb, eb + O.U * np.abs(wb), "dbeta")
