"""Plain forms in 64 bits of the gradient norm, clipping and group norm, written
from their formulas (test infrastructure; shares nothing with the kernels)."""
import math

import numpy as np

U = 2.0 ** -24  # unit roundoff of fp32
# relative rounding of a result to its type, and half the spacing of its subnormals
OUT = {"f32": (U, 2.0 ** -150), "bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25)}
EPS = float(np.float32(1e-5))


def norms(rows, off, n, inf):
    """(K,), (K, L) norms of the tensors of float64 rows."""
    parts = [[rows[k][o:o + m] for o, m in zip(off, n)] for k in range(len(rows))]
    if inf:
        t = np.array([[np.max(np.abs(p)) for p in r] for r in parts])
        return t.max(1), t
    s = np.array([[np.dot(p, p) for p in r] for r in parts])
    return np.array([math.sqrt(math.fsum(r)) for r in s]), np.sqrt(s)


def clip_factor(max_norm, norm):
    """The factor as it is defined, in fp32."""
    with np.errstate(all="ignore"):
        q = np.float32(max_norm) / (np.float32(norm) + np.float32(1e-6))
    return np.float32(1.0) if q >= 1 else q


def sigmoid(z):
    return 0.5 * (1.0 + np.tanh(0.5 * z))


def act(z, kind):
    return {"none": z, "relu": np.where(z < 0, 0.0, z), "silu": z * sigmoid(z)}[kind]


def act_grad(z, kind):
    s = sigmoid(z)
    return {"none": np.ones_like(z), "relu": (z > 0) * 1.0, "silu": s * (1 + z * (1 - s))}[kind]


def stats(x, G, eps=EPS):
    """mean and 1/sqrt(var + eps), (K, N, G), of x (K, N, P, C)."""
    K, N, P, C = x.shape
    v = x.reshape(K, N, P, G, C // G)
    mean = v.mean((2, 4))
    var = ((v - mean[:, :, None, :, None]) ** 2).mean((2, 4))
    return mean, 1.0 / np.sqrt(var + eps)


def spread(s, C):
    """(K, N, G) per group -> (K, N, 1, C)."""
    return np.repeat(s, C // s.shape[2], axis=2)[:, :, None, :]


def forward(x, gamma, beta, G, kind, eps=EPS):
    """y, mean, rstd and what bounds y's rounding: |gamma xhat| + |beta|."""
    mean, rstd = stats(x, G, eps)
    C = x.shape[3]
    h = (x - spread(mean, C)) * spread(rstd, C)
    gh, b = gamma[:, None, None, :] * h, beta[:, None, None, :]
    return act(gh + b, kind), mean, rstd, np.abs(gh) + np.abs(b)


def backward(dy, x, mean, rstd, gamma, beta, kind):
    """dx, dgamma, dbeta and bounds on their fp32 errors (see `bounds`)."""
    K, N, P, C = x.shape
    G = mean.shape[2]
    m = P * (C // G)
    r, ga = spread(rstd, C), gamma[:, None, None, :]
    h = (x - spread(mean, C)) * r
    z = ga * h + beta[:, None, None, :]
    dz = dy * act_grad(z, kind)

    def group(v):  # (K, N, P, C) -> sums per group, spread again
        return spread(v.sum(2).reshape(K, N, G, C // G).sum(3), C)

    s1, s2 = group(ga * dz) / m, group(ga * dz * h) / m
    dx = r * (ga * dz - s1 - h * s2)
    out = dx, (dz * h).sum((1, 2)), dz.sum((1, 2))
    return out, bounds(dy, h, z, dz, ga, beta, s1, s2, r, m, group)


# fp32 terms a thread adds one after another, at most
CHAIN = 64


def bounds(dy, h, z, dz, ga, beta, s1, s2, r, m, group):
    """First-order bounds with u = 2^-24.  xhat: 2 roundings.  z = fma(xhat, gamma,
    beta): |dz_| <= u (2 |gamma xhat| + |z|) <= 3 u w, w = |gamma xhat| + |beta|.  act' of
    silu: a sigmoid good to 4 u (1 + |z|) at most, slope of act' at most 1/2, 4 operations:
    |d act'| <= u (12 + 6 w).  dz = dy act': the same times |dy|, one more rounding.  A sum
    of products over a chain of CHAIN fp32 terms (the rest in binary64) adds CHAIN + 2
    roundings of its terms."""
    w = np.abs(ga * h) + np.abs(beta[:, None, None, :])
    e_dz = U * np.abs(dy) * (13 + 6 * w)
    e_h = 2 * U * np.abs(h)
    mag = np.abs(dy) * 1.1
    e_a = e_dz * np.abs(h) + mag * e_h + (CHAIN + 2) * U * mag * np.abs(h)
    e_b = e_dz + (CHAIN + 2) * U * mag
    e1 = group(np.abs(ga) * e_b) / m + U * np.abs(s1)
    e2 = group(np.abs(ga) * e_a) / m + U * np.abs(s2)
    e_dx = r * (np.abs(ga) * e_dz + e1 + np.abs(h) * e2 + np.abs(s2) * e_h
                + 4 * U * (np.abs(ga) * mag + np.abs(s1) + np.abs(h * s2)))
    return e_dx, e_a.sum((1, 2)), e_b.sum((1, 2))


def assert_within(got, want, bound, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    err = np.abs(got - want)
    ok = err <= bound
    if not ok.all():
        i = tuple(np.argwhere(~ok)[0])
        raise AssertionError(f"{what}: {int((~ok).sum())} of {ok.size} values off; first at {i}: "
                             f"got {got[i]!r} want {want[i]!r} err {err[i]:.3g} "
                             f"bound {np.broadcast_to(bound, err.shape)[i]:.3g}")
