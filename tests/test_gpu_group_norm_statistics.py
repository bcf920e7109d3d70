"""The gradient of group norm where means lie far above the deviation: it is taken at the fp32
statistics that the forward call left."""
import numpy as np
import pytest
import torch

from tests import operators_oracle as O
from tests import test_gpu_group_norm as T

pytestmark = pytest.mark.gpu


def _moved(dy, h, ga, s1, s2, r, m, group, e_h, rho, kind):
    """How far dx, dgamma and dbeta move when xhat moves by at most e_h and rstd by rho of
    itself.  z moves by |gamma| e_h, and act' by at most half of that for silu (its slope's
    bound); for none and relu (away from the kink) not at all."""
    slope = 0.5 if kind == "silu" else 0.0
    e_dz = np.abs(dy) * slope * np.abs(ga) * e_h
    mag = 1.1 * np.abs(dy)
    e_a = e_dz * (np.abs(h) + e_h) + mag * e_h
    e1, e2 = group(np.abs(ga) * e_dz) / m, group(np.abs(ga) * e_a) / m
    whole = np.abs(ga) * mag + np.abs(s1) + np.abs(h * s2)
    e_in = np.abs(ga) * e_dz + e1 + (np.abs(h) + e_h) * e2 + np.abs(s2) * e_h
    return r * (e_in + rho * (whole + e_in)), e_a.sum((1, 2)), e_dz.sum((1, 2))


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape", [(2, 2, 196, 64, 8), (1, 1, 6000, 32, 4), (2, 3, 100, 30, 5),
                                   (1, 2, 100, 441, 7)], ids=str)
def test_backward_against_64_bit_statistics(shape, act):
    """Means of about 1e4 deviations.  The stored mean errs by u |mean| (its rounding, u = 2^-24)
    and 2^-50 sqrt(E[x^2]) (the binary64 sums), so xhat moves by rstd times that and by rstd's own
    error of itself; what follows from it adds to the kernels' rounding at the stored
    statistics.  relu: dy is 0 where z lies within twice that distance of the kink."""
    print(f"[case] {shape} {act}", flush=True)
    S = T._S()
    K, N, P, C, G = shape
    x, dy, gamma, beta = T._inputs(shape, "f32", 15)
    x += 1e4
    plan = T._plan(S, shape, "f32", act)
    _, mean, rstd = T._forward(S, plan, x, gamma, beta)
    hx, hg, hb = T._np(x), T._np(gamma), T._np(beta)
    m64, r64 = O.stats(hx, G)
    sq = (hx ** 2).reshape(K, N, P, G, C // G).mean((2, 4)) + O.EPS
    dm = 1.01 * O.U * np.abs(m64) + 2.0 ** -50 * np.sqrt(sq)
    rho = O.spread(1.01 * O.U + 2.0 ** -50 * sq * r64 ** 2, C)
    r, ga = O.spread(r64, C), hg[:, None, None, :]
    h = (hx - O.spread(m64, C)) * r
    e_h = r * O.spread(dm, C) * (1 + rho) + rho * np.abs(h)
    assert 1e-4 < e_h.max() < 1e-2
    if act == "relu":
        z = ga * h + hb[:, None, None, :]
        near = np.abs(z) < 2 * np.abs(ga) * e_h + 1e-4
        assert near.mean() < 0.01
        dy.masked_fill_(torch.from_numpy(near).cuda(), 0.0)
    hd = T._np(dy)
    dx = torch.empty_like(x)
    dg, db = torch.empty((K, C), device="cuda"), torch.empty((K, C), device="cuda")
    S.saef_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, dx, dg, db)
    # the kernels' own rounding, at the statistics they were given
    _, (kx, kg, kb) = O.backward(hd, hx, T._np(mean), T._np(rstd), hg, hb, act)
    (wx, wg, wb), _ = O.backward(hd, hx, m64, r64, hg, hb, act)
    m = P * (C // G)

    def group(v):
        return O.spread(v.sum(2).reshape(K, N, G, C // G).sum(3), C)
    dz = hd * O.act_grad(ga * h + hb[:, None, None, :], act)
    s1, s2 = group(ga * dz) / m, group(ga * dz * h) / m
    mx, mg, mb = _moved(hd, h, ga, s1, s2, r, m, group, e_h, rho, act)
    for got, want, e, what in ((dx, wx, kx + mx, "dx"), (dg, wg, kg + mg, "dgamma"),
                               (db, wb, kb + mb, "dbeta")):
        O.assert_within(T._np(got), want, e + O.U * (np.abs(want) + e), what)
