"""Group norm with an activation, forward and backward, against the 64-bit formulas."""
import math

import numpy as np
import pytest
import torch

from tests import operators_oracle as O

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# (K, N, P, C, G): one value; one pixel; odd pixels and channels; channels that no vector
# divides; groups inside a vector, of one channel, of all channels; samples cut into many pixel
# ranges; channel counts above a workgroup's and odd ones above that
SHAPES = [(1, 1, 1, 1, 1), (2, 3, 1, 16, 2), (1, 2, 7, 8, 8), (3, 2, 49, 32, 4), (2, 2, 64, 64, 64),
          (1, 3, 65, 24, 3), (2, 1, 33, 30, 5), (1, 2, 50, 33, 11), (2, 2, 121, 7, 1),
          (1, 1, 12544, 16, 4), (1, 1, 3136, 12, 12), (1, 1, 5000, 9, 3), (3, 5, 196, 128, 32),
          (1, 2, 49, 2048, 32), (1, 1, 20, 4096, 32), (1, 1, 9, 4096, 4096), (1, 1, 6, 2001, 3),
          (1, 1, 3, 6150, 6), (2, 1, 40, 520, 8), (8, 16, 64, 64, 8), (1, 1, 784, 512, 32)]


def _S():
    from paper_2008_05823_amd import saef
    return saef


def _inputs(shape, dtype, seed, loc=1.0):
    """Features and dy on the device (K, N, P, C); gamma, beta as columns of wider rows."""
    K, N, P, C, G = shape
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn((K, N, P, C), generator=gen, device="cuda")
    x = (x * (0.5 + torch.rand(C, generator=gen, device="cuda"))
         + loc * torch.randn(C, generator=gen, device="cuda")).to(DT[dtype])
    dy = torch.randn((K, N, P, C), generator=gen, device="cuda").to(DT[dtype])
    pad = (C + 63) // 64 * 64
    par = torch.full((K, 2 * pad + 64), math.nan, device="cuda")  # what lies between is not read
    par[:, :C] = 1 + 0.3 * torch.randn((K, C), generator=gen, device="cuda")
    par[:, pad:pad + C] = 0.3 * torch.randn((K, C), generator=gen, device="cuda")
    return x, dy, par[:, :C], par[:, pad:pad + C]


def _np(t):
    return t.double().cpu().numpy()


def _plan(S, shape, dtype, act):
    K, N, P, C, G = shape
    return S.GroupNorm(K, N, P, C, G, DT[dtype],
                       act={"none": S.ACT_NONE, "relu": S.ACT_RELU, "silu": S.ACT_SILU}[act])


def _forward(S, plan, x, gamma, beta):
    y = torch.full_like(x, math.nan)
    mean, rstd = (torch.full((plan.K, plan.N, plan.G), math.nan, device="cuda") for _ in range(2))
    S.saef_group_norm_forward(plan, x, gamma, beta, y, mean, rstd)
    return y, mean, rstd


def _check_forward(x, gamma, beta, G, act, dtype, y, mean, rstd):
    """y: (x - mean) is rounded once, then scaled by a factor of two roundings and added to
    beta with one: 4 u |gamma xhat| + u (|beta| + |z|) + mean's own remainder (2^-48); silu
    (slope at most 1.1) and its sigmoid add 6 u |z|.  16 u (|gamma xhat| + |beta|) covers them;
    then the rounding to the type.  Statistics: binary64, rounded to fp32; cancellation
    in the variance leaves 2^-50 (mean^2 / var + 1) of it, at most, for sums this long."""
    want, wm, wr, w = O.forward(x, gamma, beta, G, act)
    rel, tiny = O.OUT[dtype]
    # the group's own statistics, whose remainder is that of E[x^2]
    K, N, P, C = x.shape
    sq = (x ** 2).reshape(K, N, P, G, C // G).mean((2, 4)) + O.EPS
    amp = 2.0 ** -50 * sq * wr ** 2
    O.assert_within(mean.cpu(), wm, O.U * 1.01 * np.abs(wm) + 2.0 ** -50 * np.sqrt(sq), "mean")
    O.assert_within(rstd.cpu(), wr, (O.U * 1.01 + amp) * wr, "rstd")
    err = 16 * O.U * w + 2 * O.spread(amp, C) * w
    # (mean's binary64 error, seen through rstd)
    err += np.abs(gamma)[:, None, None, :] * O.spread(2.0 ** -50 * np.sqrt(sq) * wr, C)
    O.assert_within(_np(y), want, err + (rel * (np.abs(want) + err)) + tiny, "y")


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, dtype, act):
    print(f"[case] {shape} {dtype} {act}", flush=True)
    S = _S()
    x, _, gamma, beta = _inputs(shape, dtype, 1)
    y, mean, rstd = _forward(S, _plan(S, shape, dtype, act), x, gamma, beta)
    _check_forward(_np(x), _np(gamma), _np(beta), shape[4], act, dtype, y, mean, rstd)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, dtype, act):
    """Bounds of operators_oracle.bounds, and the rounding to the type.  relu: dy is 0 where
    z lies within rounding of the kink."""
    print(f"[case] {shape} {dtype} {act}", flush=True)
    S = _S()
    K, N, P, C, G = shape
    x, dy, gamma, beta = _inputs(shape, dtype, 2)
    mean, rstd = (torch.from_numpy(v).float().cuda() for v in O.stats(_np(x), G))
    if act == "relu":
        z = O.spread(_np(rstd), C) * (_np(x) - O.spread(_np(mean), C)) * _np(gamma)[:, None, None]
        near = np.abs(z + _np(beta)[:, None, None]) < 1e-4
        dy.masked_fill_(torch.from_numpy(near).cuda(), 0.0)
    dx = torch.full_like(x, math.nan)
    pad = (C + 63) // 64 * 64
    g = torch.full((K, 2 * pad), -7.0, device="cuda")
    plan = _plan(S, shape, dtype, act)
    S.saef_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, dx, g[:, :C],
                               g[:, pad:pad + C])
    (wx, wg, wb), (ex, eg, eb) = O.backward(_np(dy), _np(x), _np(mean), _np(rstd), _np(gamma),
                                            _np(beta), act)
    rel, tiny = O.OUT[dtype]
    O.assert_within(_np(dx), wx, ex + rel * (np.abs(wx) + ex) + tiny, "dx")
    O.assert_within(_np(g[:, :C]), wg, eg + O.U * np.abs(wg), "dgamma")
    O.assert_within(_np(g[:, pad:pad + C]), wb, eb + O.U * np.abs(wb), "dbeta")
    # only the gradients' columns are written, and the same again
    assert bool((g[:, C:pad] == -7.0).all()) and bool((g[:, pad + C:] == -7.0).all())
    dx2, g2 = torch.empty_like(dx), torch.full_like(g, -7.0)
    S.saef_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, dx2, g2[:, :C],
                               g2[:, pad:pad + C])
    assert torch.equal(dx, dx2) and torch.equal(g, g2)


# Channels that vectors do not divide, samples small enough to stay in registers: channels that
# repeat inside a vector; within a wave; over more threads than one; one pixel; one sample a
# worker and several; a sample that just fits (2 x 256 x 4 x 4 values in f32), and one more pixel
ODD = [(2, 3, 5, 1, 1), (3, 1, 9, 2, 1), (2, 2, 31, 3, 3), (2, 4, 17, 6, 2), (3, 1, 40, 10, 5),
       (1, 5, 1, 27, 9), (2, 1, 1, 2046, 33), (4, 3, 49, 100, 10), (1, 2, 200, 63, 7),
       (2, 2, 7, 514, 2), (1, 3, 8192, 1, 1), (1, 2, 8193, 1, 1), (2, 1, 2730, 6, 3)]


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", ODD, ids=str)
def test_odd_channels(shape, dtype, act):
    test_forward(shape, dtype, act)
    test_backward(shape, dtype, act)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", [(2, 3, 31, 27, 9), (1, 2, 200, 3, 1)], ids=str)
def test_odd_channels_write_their_features_only(shape, dtype):
    """Features inside larger buffers: what lies around the inputs (NaN) is not used, what lies
    around the outputs stays."""
    S = _S()
    x, dy, gamma, beta = _inputs(shape, dtype, 12)
    plan = _plan(S, shape, dtype, "silu")
    y, mean, rstd = _forward(S, plan, x, gamma, beta)
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    S.saef_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, dx, dg, db)
    n = x.numel()

    def room(fill):
        return torch.full((n + 64,), fill, dtype=x.dtype, device="cuda")

    def inner(v):
        return v[17:17 + n].view(x.shape)
    rx, rdy, ry, rdx = room(math.nan), room(math.nan), room(-3.0), room(-3.0)
    inner(rx).copy_(x)
    inner(rdy).copy_(dy)
    mean2, rstd2, dg2, db2 = (torch.empty_like(v) for v in (mean, rstd, dg, db))
    S.saef_group_norm_forward(plan, inner(rx), gamma, beta, inner(ry), mean2, rstd2)
    S.saef_group_norm_backward(plan, inner(rdy), inner(rx), gamma, beta, mean, rstd, inner(rdx),
                               dg2, db2)
    for got, want in ((inner(ry), y), (mean2, mean), (rstd2, rstd), (inner(rdx), dx), (dg2, dg),
                      (db2, db)):
        assert torch.equal(got, want)
    for r in (ry, rdx):
        assert bool((r[:17] == -3.0).all()) and bool((r[17 + n:] == -3.0).all())


@pytest.mark.parametrize("shape", [(1, 1, 64, 8, 2), (2, 2, 196, 64, 8), (1, 1, 6000, 32, 4)],
                         ids=str)
def test_means_far_above_the_deviation(shape):
    S = _S()
    x, _, gamma, beta = _inputs(shape, "f32", 3)
    x += 1e4
    y, mean, rstd = _forward(S, _plan(S, shape, "f32", "none"), x, gamma, beta)
    _check_forward(_np(x), _np(gamma), _np(beta), shape[4], "none", "f32", y, mean, rstd)


@pytest.mark.parametrize("shape", [(1, 2, 49, 16, 2), (1, 2, 3136, 64, 4)], ids=str)
def test_constant_features(shape):
    """Zero variance: y is act(beta)."""
    S = _S()
    x, _, gamma, beta = _inputs(shape, "f32", 4)
    x.fill_(0.3)
    y, mean, rstd = _forward(S, _plan(S, shape, "f32", "none"), x, gamma, beta)
    _check_forward(_np(x), _np(gamma), _np(beta), shape[4], "none", "f32", y, mean, rstd)


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("shape", [(2, 2, 49, 16, 2), (1, 2, 3136, 64, 4)], ids=str)
def test_values_that_are_not_finite(shape, value):
    """They make their own sample and group no number, and leave the others as they are."""
    S = _S()
    K, N, P, C, G = shape
    x, dy, gamma, beta = _inputs(shape, "f32", 5)
    plan = _plan(S, shape, "f32", "silu")
    clean = _forward(S, plan, x, gamma, beta)
    x[K - 1, 1, P // 2, 0] = value
    y, mean, rstd = _forward(S, plan, x, gamma, beta)
    hit = torch.zeros((K, N, G), dtype=torch.bool, device="cuda")
    hit[K - 1, 1, 0] = True
    wide = hit.repeat_interleave(C // G, 2)[:, :, None].expand(x.shape)
    assert bool(torch.isnan(y[wide]).all()) and bool(torch.isnan(rstd[hit]).all())
    assert torch.equal(y[~wide], clean[0][~wide])
    assert torch.equal(mean[~hit], clean[1][~hit]) and torch.equal(rstd[~hit], clean[2][~hit])


@pytest.mark.parametrize("dtype", list(DT))
def test_activations_at_extremes(dtype):
    """silu and relu far from 0: no overflow on either side."""
    S = _S()
    shape = (1, 1, 64, 8, 1)
    x, _, gamma, beta = _inputs(shape, dtype, 6)
    beta.copy_(torch.tensor([-200.0, -90.0, -87.0, -30.0, 30.0, 88.0, 200.0, 3e4], device="cuda"))
    gamma.fill_(0.01)
    for act in ("relu", "silu"):
        y, mean, rstd = _forward(S, _plan(S, shape, dtype, act), x, gamma, beta)
        _check_forward(_np(x), _np(gamma), _np(beta), 1, act, dtype, y, mean, rstd)


def test_offsets_past_32_bits():
    """More than 2^31 values: the last sample as a plan for it alone gives it, to rounding."""
    S = _S()
    N, P, C, G = 33, 65536, 1024, 32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.zeros((1, N, P, C), dtype=torch.bfloat16, device="cuda")
    x[0, N - 1] = torch.randn((P, C), generator=gen, device="cuda") + 0.5
    gamma = torch.rand((1, C), generator=gen, device="cuda") + 0.5
    beta = torch.rand((1, C), generator=gen, device="cuda")
    big = S.GroupNorm(1, N, P, C, G, torch.bfloat16, act=S.ACT_RELU)
    y, mean, rstd = _forward(S, big, x, gamma, beta)
    small = S.GroupNorm(1, 1, P, C, G, torch.bfloat16, act=S.ACT_RELU)
    last = x[:, N - 1:].contiguous()
    y1, mean1, rstd1 = _forward(S, small, last, gamma, beta)
    assert torch.allclose(mean[:, N - 1:], mean1, rtol=1e-6, atol=0)
    assert torch.allclose(rstd[:, N - 1:], rstd1, rtol=1e-6, atol=0)
    off = (y[:, N - 1].float() - y1[:, 0].float()).abs() > 2.0 ** -7 * y1[:, 0].float().abs() + 1e-5
    assert not bool(off.any())
    assert bool((y[0, 0] == beta[0].bfloat16()).all())
    dx, dx1 = y, y1  # their memory is free now
    dg, db, dg1, db1 = (torch.empty((1, C), device="cuda") for _ in range(4))
    dy = torch.zeros_like(x)
    dy[0, N - 1] = torch.randn((P, C), generator=gen, device="cuda")
    S.saef_group_norm_backward(big, dy, x, gamma, beta, mean, rstd, dx, dg, db)
    S.saef_group_norm_backward(small, dy[:, N - 1:].contiguous(), last, gamma, beta,
                               mean[:, N - 1:].contiguous(), rstd[:, N - 1:].contiguous(), dx1,
                               dg1, db1)
    size = dx1.float().abs().max()
    assert float((dx[:, N - 1].float() - dx1[:, 0].float()).abs().max() / size) < 2.0 ** -7
    assert bool((dx[0, :N - 1] == 0).all())
    # sums of 65536 terms of size about 1 in another order
    assert float((dg - dg1).abs().max()) < 1e-2 and float((db - db1).abs().max()) < 1e-2
    del x, y, dy, dx
    torch.cuda.empty_cache()


def test_channels_last_tensors_and_refusals():
    S = _S()
    plan = S.GroupNorm(2, 3, 35, 16, 4, torch.float32, act=S.ACT_RELU)
    x, _, gamma, beta = _inputs((2, 3, 35, 16, 4), "f32", 8)
    y, mean, rstd = _forward(S, plan, x, gamma, beta)
    img = x.view(6, 5, 7, 16).permute(0, 3, 1, 2)  # (N, C, H, W), channels_last
    out = torch.empty_like(img, memory_format=torch.channels_last)
    S.saef_group_norm_forward(plan, img, gamma, beta, out, mean, rstd)
    assert torch.equal(out.permute(0, 2, 3, 1).reshape(y.shape), y)

    def refused(err, *a):
        with pytest.raises(err):
            S.saef_group_norm_forward(plan, *a)
    refused(ValueError, img.contiguous(), gamma, beta, out, mean, rstd)   # channels first
    refused(ValueError, x[:, :2], gamma, beta, y, mean, rstd)
    refused(ValueError, x, gamma[:1], beta, y, mean, rstd)
    refused(ValueError, x, gamma, beta.contiguous(), y, mean, rstd)       # other worker stride
    refused(ValueError, x, gamma.t().contiguous().t(), beta, y, mean, rstd)
    refused(ValueError, x, gamma, beta, y, mean[:1], rstd)
    refused(TypeError, x.half(), gamma, beta, y, mean, rstd)
    refused(TypeError, x, gamma.half(), beta, y, mean, rstd)
    refused(TypeError, x, gamma, beta, y.cpu(), mean, rstd)
    refused(S.SaefError, x, gamma, beta, x, mean, rstd)                   # in place
    refused(S.SaefError, x, gamma, beta, y, mean, mean)
    dx, dg = torch.empty_like(x), torch.zeros((2, 64), device="cuda")

    def back(err, dx, dg, db):
        with pytest.raises(err):
            S.saef_group_norm_backward(plan, y, x, gamma, beta, mean, rstd, dx, dg, db)
    back(S.SaefError, x, dg[:, :16], dg[:, 16:32])
    back(S.SaefError, y, dg[:, :16], dg[:, 16:32])
    back(S.SaefError, dx, dg[:, :16], dg[:, 8:24])
    # dbeta of one worker over dgamma of the next
    tall = torch.zeros((3, 64), device="cuda")
    back(S.SaefError, dx, tall[:2, :16], tall[1:, :16])
    back(S.SaefError, dx, tall[1:, :16], tall[:2, 8:24])
    back(S.SaefError, dx, tall[:2, 56:].as_strided((2, 16), (64, 1)), tall[1:, :16])
    S.saef_group_norm_backward(plan, y, x, gamma, beta, mean, rstd, dx, tall[:2, 48:],
                               tall[1:, :16])
    back(S.SaefError, dx, gamma, beta)
    back(ValueError, dx, dg[:, :16], dg[:1, 16:32])
    plan.destroy()
    refused(ValueError, x, gamma, beta, y, mean, rstd)
    with pytest.raises(TypeError):
        S.GroupNorm(1, 1, 1, 8, 2, torch.float64)
    with pytest.raises(S.SaefError):
        S.GroupNorm(1, 1, 1, 8, 3)


@pytest.mark.parametrize("shape", [(2, 2, 49, 64, 8), (1, 2, 3136, 64, 8)], ids=str)
def test_another_stream_and_graph_replays(shape):
    S = _S()
    K, N, P, C, G = shape
    x, dy, gamma, beta = _inputs(shape, "bf16", 9)
    plan = _plan(S, shape, "bf16", "silu")
    y, mean, rstd = _forward(S, plan, x, gamma, beta)
    dx, dg, db = torch.empty_like(x), torch.empty((K, C), device="cuda"), torch.empty(
        (K, C), device="cuda")
    outs = (y, mean, rstd, dx, dg, db)

    def work():
        S.saef_group_norm_forward(plan, x, gamma, beta, y, mean, rstd)
        S.saef_group_norm_backward(plan, dy, x, gamma, beta, mean, rstd, dx, dg, db)

    def results():
        torch.cuda.synchronize()
        got = [v.clone() for v in outs]
        for v in outs:
            v.fill_(-1.0)
        torch.cuda.synchronize()
        return got
    work()
    want = results()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        work()
    for p, q in zip(want, results()):
        assert torch.equal(p, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in range(4):
        x.mul_(1.25)
        work()
        want = results()
        graph.replay()
        for p, q in zip(want, results()):
            assert torch.equal(p, q), i


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", [(2, 2, 49, 64, 8), (1, 2, 3136, 64, 8), (1, 1, 65, 30, 5)],
                         ids=str)
def test_features_at_odd_addresses(shape, dtype):
    """Features that start one element past an alignment boundary, as slices of larger
    buffers do: aligned ones may be read another way, so the results agree to rounding."""
    S = _S()
    K, N, P, C, G = shape
    x, dy, gamma, beta = _inputs(shape, dtype, 10)
    n = x.numel()

    def odd(t=None):
        buf = torch.full((n + 9,), -5.0, dtype=DT[dtype], device="cuda")
        v = buf[1:n + 1].view(x.shape)
        if t is not None:
            v.copy_(t)
        return buf, v
    (_, xo), (_, dyo), (ybuf, yo), (dbuf, dxo) = odd(x), odd(dy), odd(), odd()
    plan = _plan(S, shape, dtype, "silu")
    mean, rstd = (torch.empty((K, N, G), device="cuda") for _ in range(2))
    S.saef_group_norm_forward(plan, xo, gamma, beta, yo, mean, rstd)
    _check_forward(_np(x), _np(gamma), _np(beta), G, "silu", dtype, yo, mean, rstd)
    dg, db = torch.empty((K, C), device="cuda"), torch.empty((K, C), device="cuda")
    S.saef_group_norm_backward(plan, dyo, xo, gamma, beta, mean, rstd, dxo, dg, db)
    (wx, wg, wb), (ex, eg, eb) = O.backward(_np(dy), _np(x), _np(mean), _np(rstd), _np(gamma),
                                            _np(beta), "silu")
    rel, tiny = O.OUT[dtype]
    O.assert_within(_np(dxo), wx, ex + rel * (np.abs(wx) + ex) + tiny, "dx")
    O.assert_within(_np(dg), wg, eg + O.U * np.abs(wg), "dgamma")
    O.assert_within(_np(db), wb, eb + O.U * np.abs(wb), "dbeta")
    for buf in (ybuf, dbuf):  # nothing around them is written
        assert float(buf[0]) == -5.0 and bool((buf[n + 1:] == -5.0).all())
