"""The 64-bit plain forms against differences, and the argument checks that need no GPU."""
import ctypes

import numpy as np
import pytest

from tests import operators_oracle as O


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 8, 1), (2, 3, 5, 12, 3), (2, 2, 9, 6, 6)])
def test_group_norm_gradient_against_differences(kind, shape):
    """d/dt L(v + t u) at 0 for L = sum(y w), by central differences of step 1e-5: their error
    is of second order, about 1e-10 times the third derivative, and rounding 1e-16 / 1e-5."""
    K, N, P, C, G = shape
    rng = np.random.default_rng(7)
    x = rng.standard_normal((K, N, P, C))
    gamma, beta = 1 + 0.3 * rng.standard_normal((2, K, C))
    w = rng.standard_normal(x.shape)
    y, mean, rstd, _ = O.forward(x, gamma, beta, G, kind)
    (dx, dg, db), _ = O.backward(w, x, mean, rstd, gamma, beta, kind)
    z = gamma[:, None, None] * (x - O.spread(mean, C)) * O.spread(rstd, C) + beta[:, None, None]
    assert kind != "relu" or np.abs(z).min() > 1e-3  # away from the kink

    def loss(a, b, c):
        return (O.forward(a, b, c, G, kind)[0] * w).sum()
    h = 1e-5
    for i, grad in enumerate((dx, dg, db)):
        for _ in range(4):
            u = rng.standard_normal(grad.shape)
            at = [x, gamma, beta]
            lo, hi = list(at), list(at)
            lo[i], hi[i] = at[i] - h * u, at[i] + h * u
            diff = (loss(*hi) - loss(*lo)) / (2 * h)
            assert abs(diff - (grad * u).sum()) <= 1e-6 * (1 + np.abs(grad * u).sum()), (i, kind)


def test_clip_factor():
    assert O.clip_factor(1.0, 0.0) == 1.0
    assert O.clip_factor(1.0, 0.999) == 1.0
    assert O.clip_factor(0.0, 3.0) == 0.0
    assert O.clip_factor(1.0, np.inf) == 0.0
    assert np.isnan(O.clip_factor(1.0, np.nan))


def test_null_handles_are_rejected():
    from paper_2008_05823_amd import saef as S
    lib, f, h = S.raw_library(), ctypes.c_float, ctypes.c_void_p()
    null = None
    assert lib.saef_grads_create(null, 1, 0, null, ctypes.byref(h)) == S.EINVAL
    assert lib.saef_grads_create(null, 1, 0, null, null) == S.EINVAL
    assert lib.saef_grads_destroy(null) == S.EINVAL
    assert lib.saef_grad_norm(null, 0, null, null, null) == S.EINVAL
    assert lib.saef_clip(null, f(1.0), null, null, null) == S.EINVAL
    assert lib.saef_round_end_clipped(null, 0, 0, 1, f(0.1), f(0), 1, f(1), *([null] * 11)) \
        == S.EINVAL
    assert lib.saef_group_norm_destroy(null) == S.EINVAL
    assert lib.saef_group_norm_forward(null, null, null, null, 4, *([null] * 4)) == S.EINVAL
    assert lib.saef_group_norm_backward(null, *([null] * 4), 4, *([null] * 5), 4, null) == S.EINVAL
    assert h.value is None


@pytest.mark.parametrize("bad", [
    dict(K=0), dict(K=4097), dict(N=0), dict(P=0), dict(C=0), dict(C=65540), dict(G=0), dict(G=3),
    dict(dtype=-1), dict(dtype=3), dict(act=-1), dict(act=3), dict(eps=0.0), dict(eps=-1.0),
    dict(eps=float("inf")), dict(eps=float("nan")), dict(P=1 << 40), dict(N=1 << 62),
    dict(K=4096, C=65536, N=1, P=1)])
def test_group_norm_shapes_are_checked(bad):
    from paper_2008_05823_amd import saef as S
    a = dict(dict(K=2, N=3, P=5, C=8, G=2, dtype=0, act=0, eps=1e-5), **bad)
    h = ctypes.c_void_p()
    assert S.raw_library().saef_group_norm_create(
        a["K"], a["N"], a["P"], a["C"], a["G"], a["dtype"], a["act"], ctypes.c_float(a["eps"]),
        ctypes.byref(h)) == S.EINVAL
    assert h.value is None
