"""Gradient norms, clipping and the clipped second half of an iteration on the GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2008_05823_amd import workloads as W
from tests import operators_oracle as O

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# tensor sizes around a tile (2048 elements), a 16-byte vector, a word, and 1; many tiny
# ones; a large one
SIZES = {"one": [1], "small": [5, 64, 1, 3], "tile": [2047, 2048, 2049, 4096, 31, 7],
         "tiny": [1 + (i * 37) % 100 for i in range(300)], "large": [300_001, 70_000, 129]}
SENTINEL = 7.25


def _S():
    from paper_2008_05823_amd import saef
    return saef


def _layout(sizes, K, shuffled=False):
    off, n, d_pad = W.custom(sizes, K=K).layout()
    off, n = [int(v) for v in off], [int(v) for v in n]
    if shuffled:  # tensors in another order than their addresses
        order = np.random.default_rng(3).permutation(len(n))
        off, n = [off[i] for i in order], [n[i] for i in order]
    return _S().Layout(off, n, d_pad, K), off, n, d_pad


def _rows(off, n, d_pad, K, dtype, seed, spread=3.0):
    """Device rows (padding SENTINEL) and the same values as float64 (padding 0)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    g = torch.full((K, d_pad), SENTINEL, dtype=DT[dtype], device="cuda")
    for o, m in zip(off, n):
        s = math.exp(spread * float(torch.rand(1, generator=gen, device="cuda")) - 4)
        g[:, o:o + m] = (s * torch.randn((K, m), generator=gen, device="cuda")).to(DT[dtype])
    h = np.zeros((K, d_pad))
    for o, m in zip(off, n):
        h[:, o:o + m] = g[:, o:o + m].double().cpu().numpy()
    return g, h


def _source(S, lay, g, off, n, src):
    """Grads over the rows, over tensors of their own, or over a bucket without gaps that
    starts one element past an alignment boundary."""
    if src == "rows":
        return S.Grads(lay, g), None
    if src == "list":
        parts = [[r[o:o + m].clone() for o, m in zip(off, n)] for r in g]
        return S.Grads(lay, parts), parts
    total = sum(n)
    bucket = torch.zeros(g.shape[0] * total + 1, dtype=g.dtype, device="cuda")
    parts, at = [], 1
    for r in g:
        parts.append([])
        for o, m in zip(off, n):
            bucket[at:at + m] = r[o:o + m]
            parts[-1].append(bucket[at:at + m])
            at += m
    return S.Grads(lay, parts), parts


def _norm(S, grads, L, inf):
    norms = torch.full((grads.K,), -1.0, device="cuda")
    tn = torch.full((grads.K, L), -1.0, device="cuda")
    S.saef_grad_norm(grads, norms, tensor_norms=tn, norm_type=math.inf if inf else 2)
    return norms, tn


@pytest.mark.parametrize("inf", [False, True], ids=["2", "inf"])
@pytest.mark.parametrize("src", ["rows", "list", "bucket"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("sizes", list(SIZES))
def test_norms(sizes, dtype, src, inf):
    """The binary64 sums err by n 2^-53 (< 1e-9 here), their rounding to fp32 by 2^-24; the
    largest magnitude is exact."""
    print(f"[case] {sizes} {dtype} {src} {inf}", flush=True)
    S, K = _S(), 3
    lay, off, n, d_pad = _layout(SIZES[sizes], K, shuffled=True)
    g, h = _rows(off, n, d_pad, K, dtype, 11)
    grads, _ = _source(S, lay, g, off, n, src)
    norms, tn = _norm(S, grads, len(n), inf)
    want, twant = O.norms(h, off, n, inf)
    rel = 0.0 if inf else O.U * (1 + 1e-7) + 1e-9
    O.assert_within(norms.cpu(), want, rel * want, "norms")
    O.assert_within(tn.cpu(), twant, rel * twant, "tensor norms")
    again, _ = _norm(S, grads, len(n), inf)
    assert torch.equal(norms, again)
    alone = torch.empty_like(norms)  # without the tensors' norms
    S.saef_grad_norm(grads, alone, norm_type=math.inf if inf else 2)
    assert torch.equal(norms, alone)


@pytest.mark.parametrize("src", ["rows", "list", "bucket"])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("sizes", list(SIZES))
def test_clip(sizes, dtype, src):
    """Bit for bit: fp32(c g), rounded to the type; one worker is short enough to stay."""
    print(f"[case] {sizes} {dtype} {src}", flush=True)
    S, K = _S(), 3
    lay, off, n, d_pad = _layout(SIZES[sizes], K, shuffled=True)
    g, h = _rows(off, n, d_pad, K, dtype, 12)
    keep = g.clone()
    grads, parts = _source(S, lay, g, off, n, src)
    norms, _ = _norm(S, grads, len(n), False)
    bound = float(norms.sort().values[1]) * 0.9
    out = torch.full((K, d_pad), SENTINEL, device="cuda")
    S.saef_clip(grads, bound, norms, out=out)
    f = [O.clip_factor(bound, v) for v in norms.cpu().numpy()]
    assert sum(v < 1 for v in f) == 2 or float(norms.min()) > bound
    want = keep.float().clone()
    for k in range(K):
        for o, m in zip(off, n):
            want[k, o:o + m] = keep[k, o:o + m].float() * float(f[k])
    # padding is not written
    mask = torch.zeros(d_pad, dtype=torch.bool, device="cuda")
    for o, m in zip(off, n):
        mask[o:o + m] = True
    assert torch.equal(out[:, mask], want[:, mask])
    assert bool((out[:, ~mask] == SENTINEL).all())
    assert torch.equal(g, keep)
    S.saef_clip(grads, bound, norms)  # in place
    for k in range(K):
        for i, (o, m) in enumerate(zip(off, n)):
            got = g[k, o:o + m] if src == "rows" else parts[k][i]
            assert torch.equal(got, want[k, o:o + m].to(DT[dtype])), (k, i)
    if src == "rows":
        assert bool((g[:, ~mask] == SENTINEL).all())


def test_bound_of_zero_and_of_more_than_the_norm():
    S = _S()
    lay, off, n, d_pad = _layout([100, 3000], 2)
    g, _ = _rows(off, n, d_pad, 2, "f32", 3)
    grads = S.Grads(lay, g)
    norms, _ = _norm(S, grads, 2, False)
    out = torch.full((2, d_pad), SENTINEL, device="cuda")
    S.saef_clip(grads, 1e30, norms, out=out)
    assert torch.equal(out, g)
    S.saef_clip(grads, 0.0, norms, out=out)
    assert bool((out[:, :100] == 0).all()) and bool((out[:, 128:3128] == 0).all())
    # a gradient of zeros has norm 0 and stays
    g.zero_()
    norms, tn = _norm(S, grads, 2, False)
    assert bool((norms == 0).all()) and bool((tn == 0).all())
    S.saef_clip(grads, 1.0, norms, out=out)
    assert bool((out[:, :100] == 0).all())


@pytest.mark.parametrize("inf", [False, True], ids=["2", "inf"])
@pytest.mark.parametrize("at", [0, 2100, 4999])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite(value, at, inf):
    """They reach their own worker's and tensor's norm, and nobody else's."""
    S = _S()
    lay, off, n, d_pad = _layout([64, 5000, 300], 3)
    g, h = _rows(off, n, d_pad, 3, "f32", 5)
    clean, tclean = _norm(S, S.Grads(lay, g), 3, inf)
    g[1, off[1] + at] = value
    grads = S.Grads(lay, g)
    norms, tn = _norm(S, grads, 3, inf)
    for k in range(3):
        for l in range(3):
            if (k, l) != (1, 1):
                assert tn[k, l] == tclean[k, l]
    bad = math.isnan if math.isnan(value) else math.isinf
    assert bad(float(norms[1])) and bad(float(tn[1, 1]))
    assert norms[0] == clean[0] and norms[2] == clean[2]
    out = torch.zeros((3, d_pad), device="cuda")
    S.saef_clip(grads, 1e-3, norms, out=out)
    assert math.isnan(float(out[1, off[1] + at]))
    assert bool(torch.isfinite(out[[0, 2]]).all())
    rest = out[1, off[0]:off[0] + 64]
    assert bool(torch.isnan(rest).all() if math.isnan(value) else (rest == 0).all())


def test_large_squares_neither_overflow_nor_vanish():
    S = _S()
    lay, off, n, d_pad = _layout([4000], 2)
    g = torch.zeros((2, d_pad), device="cuda")
    g[0, :4000], g[1, :4000] = 1e30, 1e-30
    norms, _ = _norm(S, S.Grads(lay, g), 1, False)
    want = np.float64(np.float32([1e30, 1e-30])) * math.sqrt(4000)
    O.assert_within(norms.cpu(), want, O.U * 1.01 * want, "norms")


def test_offsets_past_32_bits():
    """9 rows of 2^28: the last rows start beyond 2^31 elements."""
    S, K, n = _S(), 9, 1 << 28
    lay = S.Layout([0], [n], n, K)
    g = torch.zeros((K, n), dtype=torch.bfloat16, device="cuda")
    g[8] = 1.0
    g[7, n - 1] = -3.0
    grads = S.Grads(lay, g)
    norms, tn = _norm(S, grads, 1, False)
    assert norms.tolist() == [0.0] * 7 + [3.0, 16384.0] and torch.equal(tn[:, 0], norms)
    out = torch.zeros((K, n), device="cuda")
    S.saef_clip(grads, 1.0, norms, out=out)
    f = [float(O.clip_factor(1.0, v)) for v in (3.0, 16384.0)]
    assert float(out[7, n - 1]) == -3.0 * float(np.float32(f[0])) or \
        float(out[7, n - 1]) == float(np.float32(-3.0) * np.float32(f[0]))
    assert bool((out[8] == f[1]).all()) and bool((out[:7] == 0).all())
    S.saef_clip(grads, 1.0, norms)
    assert bool((g[8] == torch.tensor(f[1]).bfloat16().cuda()).all())
    del g, out
    torch.cuda.empty_cache()


def _state(w, d_pad, seed, mu, mode):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    K, W64 = w.K, d_pad // 64

    def rnd(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    return {"m": rnd(K, d_pad) if mu else None, "e": rnd(K, d_pad), "e_srv": rnd(d_pad),
            "x": rnd(d_pad),
            "signs": torch.randint(-2 ** 62, 2 ** 62, (K, W64), generator=gen, device="cuda"),
            "scales": rnd(K, w.L).abs(),
            "srv_signs": torch.randint(-2 ** 62, 2 ** 62, (W64,), generator=gen, device="cuda"),
            "srv_scales": rnd(w.L).abs()}


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("mu", [0.0, 0.9])
@pytest.mark.parametrize("t,period", [(0, 0), (3, 0), (3, 4)])
@pytest.mark.parametrize("sizes", ["small", "tile", "tiny", "large"])
def test_clipped_half_equals_clip_then_half(sizes, t, period, mu, mode):
    """saef_round_end_clipped leaves, bit for bit, what saef_clip into rows and
    saef_round_end leave, and does not touch g."""
    print(f"[case] {sizes} t={t} p={period} mu={mu} mode={mode}", flush=True)
    S = _S()
    w = W.custom(SIZES[sizes], K=3)
    lay, off, n, d_pad = _layout(SIZES[sizes], 3)
    g, _ = _rows(off, n, d_pad, 3, "f32", 21)
    keep = g.clone()
    norms, _ = _norm(S, S.Grads(lay, g), len(n), False)
    bound = float(norms.sort().values[1]) * 0.9
    a = _state(w, d_pad, 5, mu, mode)
    b = {k: None if v is None else v.clone() for k, v in a.items()}
    rows = torch.zeros_like(g)
    S.saef_clip(S.Grads(lay, g), bound, norms, out=rows)
    order = ("m", "e", "e_srv", "x", "signs", "scales", "srv_signs", "srv_scales")
    S.saef_round_end(lay, t, period, 3, 0.1, mu, mode, rows, *[a[k] for k in order])
    S.saef_round_end_clipped(lay, t, period, 3, 0.1, mu, mode, bound, norms, g,
                             *[b[k] for k in order])
    mask = torch.zeros(d_pad, dtype=torch.bool, device="cuda")
    for o, m in zip(off, n):
        mask[o:o + m] = True
    for k in order:
        if a[k] is None:
            continue
        same = a[k] == b[k]
        if k in ("m", "e", "e_srv", "x"):
            same = same[..., mask]
        assert bool(same.all()), k
    assert torch.equal(g, keep)
    assert S.saef_status(lay) == S.OK


def test_worker_without_a_norm_is_reported():
    S = _S()
    w = W.custom([5000], K=2)
    lay, off, n, d_pad = _layout([5000], 2)
    g, _ = _rows(off, n, d_pad, 2, "f32", 2)
    g[0, 17] = math.nan
    norms, _ = _norm(S, S.Grads(lay, g), 1, False)
    a = _state(w, d_pad, 5, 0.0, 1)
    order = ("m", "e", "e_srv", "x", "signs", "scales", "srv_signs", "srv_scales")
    S.saef_round_end_clipped(lay, 0, 0, 2, 0.1, 0.0, 1, 1.0, norms, g, *[a[k] for k in order])
    assert S.saef_status(lay) == S.ERANGE


def test_refusals():
    S = _S()
    lay, off, n, d_pad = _layout([100, 3000], 2)
    g = torch.zeros((2, d_pad), device="cuda")
    norms = torch.zeros(2, device="cuda")
    with pytest.raises(ValueError):
        S.Grads(lay, g[:, :-64])                       # not rows of this layout
    with pytest.raises(ValueError):
        S.Grads(lay, [[g[0, :100]]])                   # one tensor missing
    with pytest.raises(ValueError):
        S.Grads(lay, [[g[0, :100], g[0, 128:3000]]])   # a wrong size
    with pytest.raises(TypeError):
        S.Grads(lay, g.double())
    with pytest.raises(TypeError):
        S.Grads(lay, g.cpu())
    with pytest.raises(TypeError):                     # mixed types
        S.Grads(lay, [[g[0, :100], g[0, 128:3128].half()]])
    with pytest.raises(ValueError):                    # strided
        S.Grads(lay, [[g[0, :200:2], g[0, 128:3128]]])
    with pytest.raises(S.SaefError) as e:              # overlapping gradients
        S.Grads(lay, [[g[0, :100], g[0, 50:3050]]])
    assert e.value.rc == S.EINVAL
    with pytest.raises(S.SaefError):                   # more workers than the layout's
        S.Grads(lay, torch.zeros((3, d_pad), device="cuda"))
    grads = S.Grads(lay, g)
    with pytest.raises(ValueError):
        S.saef_grad_norm(grads, norms, norm_type=1)
    with pytest.raises(ValueError):
        S.saef_grad_norm(grads, norms[:1])
    with pytest.raises(ValueError):
        S.saef_grad_norm(grads, norms, tensor_norms=norms)
    out = torch.zeros((2, d_pad), device="cuda")
    for bad in (-1.0, math.nan, math.inf):
        with pytest.raises(S.SaefError):
            S.saef_clip(grads, bad, norms, out=out)
    with pytest.raises(ValueError):
        S.saef_clip(grads, 1.0, norms, out=out[:1])
    with pytest.raises(S.SaefError):
        S.saef_clip(grads, 1.0, norms, out=g)          # rows over the gradients
    with pytest.raises(S.SaefError):
        S.saef_grad_norm(grads, g[0, :2])              # norms inside the gradients
    lib, s = S.raw_library(), torch.cuda.current_stream().cuda_stream
    assert lib.saef_grad_norm(grads.handle, 2, norms.data_ptr(), None, s) == S.EINVAL
    assert lib.saef_grad_norm(grads.handle, 0, None, None, s) == S.EINVAL
    assert lib.saef_grad_norm(grads.handle, 0, norms.data_ptr() + 2, None, s) == S.EINVAL
    assert lib.saef_clip(grads.handle, 1.0, None, None, s) == S.EINVAL
    a = _state(W.custom([100, 3000], K=2), d_pad, 1, 0.0, 1)
    order = ("m", "e", "e_srv", "x", "signs", "scales", "srv_signs", "srv_scales")
    before = {k: None if v is None else v.clone() for k, v in a.items()}
    for bound, nv in ((-1.0, norms), (1.0, None), (1.0, a["scales"][:, 0].contiguous()),
                      (1.0, a["x"][:2])):
        if nv is not None and nv is not norms and nv.data_ptr() != a["x"].data_ptr():
            nv = a["scales"].view(-1)[:2]              # norms inside the scales
        with pytest.raises((S.SaefError, TypeError)):
            S.saef_round_end_clipped(lay, 1, 0, 2, 0.1, 0.0, 1, bound, nv, g,
                                     *[a[k] for k in order])
    with pytest.raises(S.SaefError):                   # momentum constant without momentum
        S.saef_round_end_clipped(lay, 1, 0, 2, 0.1, 0.9, 1, 1.0, norms, g, *[a[k] for k in order])
    torch.cuda.synchronize()
    for k, v in before.items():
        assert v is None or torch.equal(v, a[k]), k


def test_another_stream_and_graph_replays():
    """The three calls on a stream of their own, then captured; each replay against the
    eager result, with eager work in between."""
    S = _S()
    sizes = SIZES["large"]
    w = W.custom(sizes, K=3)
    lay, off, n, d_pad = _layout(sizes, 3)
    g, _ = _rows(off, n, d_pad, 3, "f32", 33)
    grads = S.Grads(lay, g)
    norms, tn = torch.zeros(3, device="cuda"), torch.zeros((3, len(n)), device="cuda")
    rows = torch.zeros_like(g)
    order = ("m", "e", "e_srv", "x", "signs", "scales", "srv_signs", "srv_scales")
    a = _state(w, d_pad, 9, 0.0, 1)
    start = {k: None if v is None else v.clone() for k, v in a.items()}

    def reset():
        for k, v in start.items():
            if v is not None:
                a[k].copy_(v)

    def work():
        S.saef_grad_norm(grads, norms, tensor_norms=tn)
        S.saef_clip(grads, 0.01, norms, out=rows)
        S.saef_round_end_clipped(lay, 2, 0, 3, 0.1, 0.0, 1, 0.01, norms, g,
                                 *[a[k] for k in order])

    def results():
        torch.cuda.synchronize()
        return [v.clone() for v in (norms, tn, rows, a["e"], a["signs"], a["scales"], a["x"])]
    work()
    want = results()
    side = torch.cuda.Stream()
    reset()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        work()
    for p, q in zip(want, results()):
        assert torch.equal(p, q)
    graph = torch.cuda.CUDAGraph()
    reset()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        work()
    for i in range(4):
        scale = 1.0 + i
        g.mul_(scale)
        reset()
        work()
        want = results()
        reset()
        for v in (norms, tn, rows):
            v.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        for p, q, in zip(want, results()):
            # padding of rows was refilled
            same = p == q
            if p.shape == rows.shape and p.dtype == rows.dtype and not bool(same.all()):
                mask = torch.zeros(d_pad, dtype=torch.bool, device="cuda")
                for o, m in zip(off, n):
                    mask[o:o + m] = True
                same = same[:, mask]
            assert bool(same.all()), i


def test_more_tensors_than_a_launch_takes_is_refused():
    """4096 workers of 4200 one-element tensors: 17.2 M (tensor, worker) pairs, a workgroup
    of 256 threads each, are more threads than a launch may have."""
    S = _S()
    L, K = 4200, 4096
    lay = S.Layout([64 * i for i in range(L)], [1] * L, 64 * L, K)
    base = torch.zeros(L * K, device="cuda")
    p = base.data_ptr()
    table = (ctypes.c_void_p * (L * K))(*range(p, p + 4 * L * K, 4))
    handle = ctypes.c_void_p()
    rc = S.raw_library().saef_grads_create(lay.handle, K, 0, table, ctypes.byref(handle))
    assert rc == S.EINVAL and handle.value is None
