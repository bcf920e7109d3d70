"""The gradient side of a worker's step, as operators that can be timed and compared.

Between the evaluation points ``saef_round_begin`` writes and the messages
``saef_round_end`` sends, a program that trains K workers takes these steps:

  gn_fwd   group norm with an activation over channels-last features, for K
           workers whose gamma and beta lie in the rows of their own evaluation points
  gn_bwd   its gradient; dgamma and dbeta go into the workers' gradient rows
  norm     each worker's global gradient norm over all of its tensors
  clip     the norm, then the gradients scaled to at most max_norm: into the
           fp32 rows of the layout, or in place
  step     the iteration's second half on gradients that are clipped as they are read

Gradients lie in the rows of a flat layout ("rows") or in one tensor per parameter, as
autograd leaves them ("list"); a list that is clipped in place is one of views into a bucket
without gaps, so that its tensors start at odd places.  Tensor lists are the model shapes of ``workloads`` or
"ragged": L tensors of odd sizes adding up to about d.
"""
import functools
import math
import random

import torch

own = False

LR = 0.1
EPS = 1e-5          # of the group norm
TINY = 1e-6         # added to the norm that max_norm is divided by
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

# d, L and sizes of the model shapes (parameter order of the usual definitions)
_FLAT = {"flat64k": (1 << 16,), "flat256m": (1 << 28,)}


def _grad(name, op, tensors, K, *, dtype="f32", src="rows", d=0, L=0, dist="normal", p="2",
          per_tensor=False, out="rows", mu=0.0):
    c = {"op": op, "tensors": tensors, "K": K, "dtype": dtype, "src": src, "d": d, "L": L,
         "dist": dist, "p": p, "per_tensor": per_tensor, "out": out, "mu": mu}
    return {"name": name, **c} if name else c


def _gn(name, op, K, N, P, C, G, *, dtype="f32", act="relu"):
    c = {"op": op, "K": K, "N": N, "P": P, "C": C, "G": G, "dtype": dtype, "act": act}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one small tensor, a handful of workers: launches and latency
        _grad("norm_flat64k_k4", "norm", "flat64k", 4),
        # the largest tensor a layout takes: nothing but reading it
        _grad("norm_flat256m_k8", "norm", "flat256m", 8),
        # the CIFAR experiments as autograd leaves them: 167 mostly tiny tensors a worker,
        # with the norm of each tensor, which training logs
        _grad("clip_resnet56_list_k8", "clip", "resnet56", 8, src="list", per_tensor=True),
        # a large model trained in 16 bits: gradients in separate tensors, heavy tails
        _grad("clip_bert_base_bf16_list_k4", "clip", "bert_base", 4, dtype="bf16", src="list",
              dist="normal_outliers"),
        # rows of ragged tensors clipped where they are, a worker count that is no power of two
        _grad("clip_ragged_inplace_k5", "clip", "ragged", 5, d=9_000_001, L=37, out="same"),
        # the CIFAR experiments' iteration: short dependent kernels
        _grad("step_resnet56_k8", "step", "resnet56", 8),
        # the ImageNet experiments' iteration with momentum
        _grad("step_resnet50_momentum_k8", "step", "resnet50", 8, dist="laplace_zeros", mu=0.9),
        # the last stage of the CIFAR network on one image: launches and latency
        _gn("gn_fwd_8x8x64_n1", "gn_fwd", 1, 1, 64, 64, 8),
        # the first stage of the CIFAR network, total batch 128 over 8 workers
        _gn("gn_fwd_32x32x16_k8", "gn_fwd", 8, 16, 1024, 16, 4),
        # the ImageNet network's stem, total batch 256 over 8 workers: images too large to keep on chip
        _gn("gn_fwd_112x112x64_bf16_k8", "gn_fwd", 8, 32, 12544, 64, 32, dtype="bf16"),
        # the middle stage of the CIFAR network, backward
        _gn("gn_bwd_16x16x32_k8", "gn_bwd", 8, 16, 256, 32, 8),
        # the ImageNet network's third stage, backward, total batch 256 over 8 workers
        _gn("gn_bwd_14x14x1024_bf16_k8", "gn_bwd", 8, 32, 196, 1024, 32, dtype="bf16", act="silu"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "clip", "step", "gn_fwd", "gn_bwd"])
    if op in ("gn_fwd", "gn_bwd"):
        K = rng.choice([1, 2, 3, 5, 8])
        G = rng.choice([1, 2, 4, 7, 8, 16, 32])
        C = G * _log_int(rng, 1, min(64, 2048 // G))
        # groups of at least 16 values: of fewer, the gradient is mostly rounding
        P = _log_int(rng, -(-16 * G // C), 12544)
        # at most the elements of the largest listed case, half of them backward
        most = (1.0e8 if op == "gn_bwd" else 2.0e8) / (K * P * C)
        N = _log_int(rng, 1, max(1.0, min(64.0, most)))
        return _gn(None, op, K, N, P, C, G, dtype=rng.choice(["f32", "bf16", "f16"]),
                   act=rng.choice(["none", "relu", "silu"]))
    K = rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16])
    if rng.random() < 0.25:
        tensors, d, L = rng.choice(["resnet56", "resnet50"]), 0, 0
    else:
        most = 4.0e8 / K
        d = _log_int(rng, 60_000, min(60_000_000.0, most))
        tensors, L = "ragged", _log_int(rng, 1, 120)
    dist = rng.choice(["normal", "laplace_zeros", "normal_outliers"])
    if op == "step":
        return _grad(None, op, tensors, K, d=d, L=L, dist=dist, mu=rng.choice([0.0, 0.0, 0.9]))
    return _grad(None, op, tensors, K, d=d, L=L, dist=dist,
                 dtype=rng.choice(["f32", "bf16", "f16"]), src=rng.choice(["rows", "list"]),
                 p=rng.choice(["2", "2", "2", "inf"]), per_tensor=rng.random() < 0.5,
                 out=rng.choice(["rows", "same"]) if op == "clip" else "rows")


# ------------------------------------------------------------------ layouts

@functools.lru_cache(maxsize=64)
def _sizes(tensors, d, L):
    if tensors in _FLAT:
        return _FLAT[tensors]
    if tensors == "resnet56":
        n = [432, 16, 16]
        c_in = 16
        for c in (16, 32, 64):
            for _ in range(9):
                n += [9 * c_in * c, c, c, 9 * c * c, c, c]
                c_in = c
        return tuple(n + [640, 10])
    if tensors == "resnet50":
        n = [9408, 64, 64]
        c_in = 64
        for w, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
            for b in range(blocks):
                n += [c_in * w, w, w, 9 * w * w, w, w, 4 * w * w, 4 * w, 4 * w]
                n += [4 * c_in * w, 4 * w, 4 * w] if b == 0 else []
                c_in = 4 * w
        return tuple(n + [2048 * 1000, 1000])
    if tensors == "bert_base":
        h, f = 768, 4 * 768
        n = [30522 * h, 512 * h, 2 * h, h, h]
        for _ in range(12):
            n += [h * h, h] * 4 + [h, h, h * f, f, f * h, h, h, h]
        return tuple(n + [h * h, h])
    r = random.Random(1000 * d + L)
    share = [math.exp(r.gauss(0.0, 1.8)) for _ in range(L)]
    total = sum(share)
    return tuple(max(1, int(d * s / total)) for s in share)


class _Layout:
    """Offsets and sizes of a case's tensors (each on a 64-element boundary)."""

    def __init__(self, case):
        self.n = list(_sizes(case["tensors"], case["d"], case["L"]))
        self.off, at = [], 0
        for n in self.n:
            self.off.append(at)
            at += (n + 63) // 64 * 64
        self.d_pad, self.d, self.L = at, sum(self.n), len(self.n)

    def per_element(self, values):
        """(..., L) values spread over their tensors' elements, 0 on padding."""
        reps = torch.tensor([v for n in self.n for v in (n, (n + 63) // 64 * 64 - n)],
                            device=values.device)
        vals = torch.stack([values, torch.zeros_like(values)], -1).flatten(-2)
        return torch.repeat_interleave(vals, reps, dim=-1, output_size=self.d_pad)

    def slices(self, rows):
        return [rows[..., o:o + n] for o, n in zip(self.off, self.n)]


# ------------------------------------------------------------------ inputs

def _fill(out, dist, scale, gen):
    """One row of gradients: `scale` per element, 0 on padding."""
    if dist == "laplace_zeros":
        out.exponential_(generator=gen)
        u = torch.rand(out.shape, generator=gen, device=out.device)
        out *= torch.where(u < 0.475, -1.0, torch.where(u < 0.95, 1.0, 0.0))
    else:
        out.normal_(generator=gen)
        if dist == "normal_outliers":
            u = torch.rand(out.shape, generator=gen, device=out.device)
            out.copy_(torch.where(u < 0.005, -100.0, torch.where(u < 0.01, 100.0, out)))
    out *= scale
    return out


def _grad_inputs(case, seed):
    """(layout, gradient rows in the case's type, factor of every worker's size)."""
    lay, K = _Layout(case), case["K"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    u = torch.rand(lay.L, generator=gen, device="cuda")
    # per-tensor sizes over three decades, worker sizes over a factor of about 4
    scale = lay.per_element(torch.exp(math.log(1e-4) + u * math.log(1e3)))
    size = torch.exp(0.35 * torch.randn(K, generator=gen, device="cuda"))
    g = torch.empty((K, lay.d_pad), dtype=DTYPES[case["dtype"]], device="cuda")
    row = torch.empty(lay.d_pad, device="cuda")
    for k in range(K):
        g[k] = _fill(row, case["dist"], scale, gen) * size[k]
    return lay, g, gen


def _prepare_grad(case, seed):
    lay, g, gen = _grad_inputs(case, seed)
    K = case["K"]
    s = {"case": case, "lay": lay, "g": g}
    norms = torch.stack([torch.linalg.vector_norm(r.float(), 2 if case["p"] == "2" else math.inf)
                         for r in g])
    # every worker's gradient is too long, the longest ones by the most
    s["max_norm"] = 0.8 * float(norms.min())
    if case["op"] == "step":
        s["norms"] = norms
        rnd = torch.randn((2, lay.d_pad), generator=gen, device="cuda")
        mask = lay.per_element(torch.ones(lay.L, device="cuda"))
        s["x"], s["e_srv"] = 0.05 * rnd[0] * mask, 0.01 * rnd[1] * mask
        s["e"] = torch.empty((K, lay.d_pad), device="cuda")
        for k in range(K):
            torch.mul(g[k].roll(1), 0.3 * mask, out=s["e"][k])
        s["m"] = g.flip(0).mul_(2.0) if case["mu"] else None
        # the middle of a run: errors and weights with their last correction pending
        words = (K + 1, lay.d_pad // 64)
        bits = torch.randint(-2 ** 63, 2 ** 63 - 1, words, generator=gen, device="cuda")
        bits &= _words(mask[None] > 0)
        s["signs"], s["srv_signs"] = bits[:K].contiguous(), bits[K].clone()
        sc = torch.rand((K + 1, lay.L), generator=gen, device="cuda") * 1e-3
        s["scales"], s["srv_scales"] = sc[:K].contiguous(), sc[K].clone()
        s["t"] = 1
    else:
        if case["src"] == "list":
            if case["op"] == "clip" and case["out"] == "same":
                s["bucket"] = torch.stack([torch.cat(lay.slices(r)) for r in g])
                s["list"] = [list(r.split(lay.n)) for r in s["bucket"]]
            else:
                s["list"] = [[v.clone() for v in lay.slices(r)] for r in g]
            s["g"] = None
        if case["op"] == "clip" and case["out"] == "rows":
            s["rows"] = torch.zeros((K, lay.d_pad), device="cuda")
    if own:
        from paper_2008_05823_amd import saef as S
        s["S"] = S
        s["layout"] = S.Layout(lay.off, lay.n, lay.d_pad, K)
        if case["op"] != "step":
            s["grads"] = S.Grads(s["layout"], s["g"] if case["src"] == "rows" else s["list"])
            s["norms"] = torch.zeros(K, device="cuda")
            s["tnorms"] = torch.zeros((K, lay.L), device="cuda") if case["per_tensor"] else None
    return s


def _gn_inputs(case, seed):
    """x, the workers' parameter rows (gamma, then beta on the next 64-element boundary), dy."""
    K, N, P, C, G = (case[k] for k in ("K", "N", "P", "C", "G"))
    dt = DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    # features with a mean and a size of their own per channel
    loc = torch.randn(C, generator=gen, device="cuda")
    size = torch.exp(0.5 * torch.randn(C, generator=gen, device="cuda"))
    x = torch.empty((K, N, P, C), dtype=dt, device="cuda")
    dy = torch.empty_like(x) if case["op"] == "gn_bwd" else None
    for k in range(K):
        x[k] = torch.randn((N, P, C), generator=gen, device="cuda") * size + loc
        if dy is not None:
            dy[k] = torch.randn((N, P, C), generator=gen, device="cuda") / N
    pad = (C + 63) // 64 * 64
    par = torch.zeros((K, 2 * pad), device="cuda")
    par[:, :C] = 1.0 + 0.2 * torch.randn((K, C), generator=gen, device="cuda")
    par[:, pad:pad + C] = 0.2 * torch.randn((K, C), generator=gen, device="cuda")
    return x, par, par[:, :C], par[:, pad:pad + C], dy


def _gn_stats(x, G):
    """mean and 1/sqrt(var + eps) per sample and group, (K, N, G), in x's own type."""
    K, N, P, C = x.shape
    v = x.view(K, N, P, G, C // G)
    mean = v.mean((2, 4))
    var = ((v - mean[:, :, None, :, None]) ** 2).mean((2, 4))
    return mean, 1.0 / torch.sqrt(var + EPS)


def _gn_saved(case, x, gamma, beta, dy):
    """What the forward pass left: the statistics.  relu: dy is 0 where the pre-activation
    lies within rounding of the kink, where the derivative is not one number."""
    stats = [_gn_stats(v[None].float(), case["G"]) for v in x]
    mean, rstd = torch.cat([a for a, _ in stats]), torch.cat([b for _, b in stats])
    if case["act"] == "relu":
        for k in range(case["K"]):
            z = _gn_z(x[k:k + 1].float(), mean[k:k + 1], rstd[k:k + 1], gamma[k:k + 1],
                      beta[k:k + 1])[1]
            dy[k].masked_fill_(z[0].abs() < 1e-3, 0.0)
    return mean, rstd


def _prepare_gn(case, seed):
    K, N, P, C, G = (case[k] for k in ("K", "N", "P", "C", "G"))
    x, par, gamma, beta, dy = _gn_inputs(case, seed)
    s = {"case": case, "x": x, "par": par, "gamma": gamma, "beta": beta}
    s["out"] = torch.empty_like(x)
    if case["op"] == "gn_bwd":
        s["dy"] = dy
        s["mean"], s["rstd"] = _gn_saved(case, x, gamma, beta, dy)
        s["gpar"] = torch.zeros_like(par)
    else:
        s["mean"], s["rstd"] = (torch.empty((K, N, G), device="cuda") for _ in range(2))
    if own:
        from paper_2008_05823_amd import saef as S
        s["S"] = S
        acts = {"none": S.ACT_NONE, "relu": S.ACT_RELU, "silu": S.ACT_SILU}
        s["plan"] = S.GroupNorm(K, N, P, C, G, x.dtype, act=acts[case["act"]], eps=EPS)
    return s


def prepare(case, seed):
    return (_prepare_gn if case["op"].startswith("gn") else _prepare_grad)(case, seed)


# ------------------------------------------------------------------ plain forms

def _plain_norm(s):
    """Per worker: the norm over all tensors and, when asked for, of each tensor."""
    c, lay = s["case"], s["lay"]
    norms, tensor_norms = [], []
    for k in range(c["K"]):
        if c["src"] == "rows" and not c["per_tensor"]:
            # padding is 0
            parts = [s["g"][k]]
        else:
            parts = lay.slices(s["g"][k]) if c["src"] == "rows" else s["list"][k]
        if c["p"] == "2":
            sums = torch.stack([v.float().square().sum() for v in parts])
            norms.append(sums.sum().sqrt())
            tensor_norms.append(sums.sqrt())
        else:
            tops = torch.stack([v.abs().max().float() for v in parts])
            norms.append(tops.max())
            tensor_norms.append(tops)
    out = {"norms": torch.stack(norms)}
    if c["per_tensor"]:
        out["tensor_norms"] = torch.stack(tensor_norms)
    return out


def _factors(max_norm, norms):
    return torch.clamp(torch.div(torch.full_like(norms, max_norm), norms + TINY), max=1.0)


def _plain_clip(s, max_norm):
    c, lay = s["case"], s["lay"]
    out = _plain_norm(s)
    f = _factors(max_norm, out["norms"])
    if c["src"] == "rows":
        y = s["g"] if c["out"] == "same" else s["rows"]
        y.copy_(s["g"].float() * f[:, None])
        out["clipped"] = y
    else:
        for k in range(c["K"]):
            to = s["list"][k] if c["out"] == "same" else lay.slices(s["rows"][k])
            for v, w in zip(s["list"][k], to):
                w.copy_(v.float() * f[k])
        out["clipped"] = s["bucket"] if c["out"] == "same" else s["rows"]
    return out


_SHIFTS = None


def _words(bits):
    """Sign words: bit b of word j is element 64 j + b."""
    global _SHIFTS
    if _SHIFTS is None or _SHIFTS.device != bits.device:
        _SHIFTS = torch.arange(64, device=bits.device)
    return (bits.view(*bits.shape[:-1], -1, 64).long() << _SHIFTS).sum(-1)


def _decode(lay, words, scales):
    """The message's values, +-scale of the tensor by the bit (padding: 0)."""
    bits = ((words[..., None] >> _SHIFTS) & 1).flatten(-2) > 0
    s = lay.per_element(scales)
    return torch.where(bits, s, -s)


def _compress(lay, delta):
    """Sign words and layer-wise scales |v|_1 / n of the rows of delta (padding: 0).  The
    sums are the method's exact ones, so they are taken in 64 bits."""
    mask = lay.per_element(torch.ones(lay.L, device=delta.device)) > 0
    l1 = torch.stack([v.abs().sum(-1, dtype=torch.float64) / v.shape[-1]
                      for v in lay.slices(delta)], -1)
    return _words((delta >= 0) & mask), l1.float()


def _plain_step(s):
    """saef_round_end's arithmetic on clipped gradients, double-way, corrections pending.
    Delta is defined with one rounding (a fused multiply-add), which decides its sign where it
    is near 0: the product and sum are taken in 64 bits, where the product is exact."""
    c, lay, K = s["case"], s["lay"], s["case"]["K"]
    f = _factors(s["max_norm"], s["norms"])
    lr, mu = (float(torch.tensor(v, dtype=torch.float32)) for v in (LR, c["mu"]))
    mean = torch.zeros(lay.d_pad, dtype=torch.float64, device="cuda")
    words, scales = [], []
    for k in range(K):
        e = s["e"][k] - _decode(lay, s["signs"][k], s["scales"][k])
        step = s["g"][k] * f[k]
        if s["m"] is not None:
            step = (s["m"][k].double() * mu + step).float()
            s["m"][k] = step
        s["e"][k] = (step.double() * lr + e).float()
        w, sc = _compress(lay, s["e"][k])
        words.append(w)
        scales.append(sc)
        mean += _decode(lay, w, sc)
    mean = (mean / K).float()
    old = _decode(lay, s["srv_signs"], s["srv_scales"])
    s["signs"].copy_(torch.stack(words))
    s["scales"].copy_(torch.stack(scales))
    s["x"] -= old
    s["e_srv"] -= old
    s["e_srv"] += mean
    w, sc = _compress(lay, s["e_srv"])
    s["srv_signs"].copy_(w)
    s["srv_scales"].copy_(sc)


def _step_out(s):
    keys = ("e", "signs", "scales", "e_srv", "srv_signs", "srv_scales", "x")
    out = {k: s[k] for k in keys}
    if s["m"] is not None:
        out["m"] = s["m"]
    return out


def _gn_z(x, mean, rstd, gamma, beta):
    """xhat and the pre-activation, in x's type; x (K, N, P, C)."""
    K, N, P, C = x.shape
    G = mean.shape[2]
    v = x.view(K, N, P, G, C // G)
    xh = ((v - mean[:, :, None, :, None]) * rstd[:, :, None, :, None]).view(K, N, P, C)
    return xh, xh * gamma[:, None, None, :] + beta[:, None, None, :]


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _act_grad(z, act):
    """The activation's derivative, None where it is 1."""
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        sg = 1 / (1 + torch.exp(-z))
        return sg * (1 + z * (1 - sg))
    return None


def _gn_backward(dy, x, mean, rstd, gamma, beta, act):
    """dx, dgamma, dbeta in x's type; x, dy (K, N, P, C)."""
    K, N, P, C = x.shape
    G = mean.shape[2]
    xh, z = _gn_z(x, mean, rstd, gamma, beta)
    d = _act_grad(z, act)
    dz = dy if d is None else dy * d
    A, B = (dz * xh).sum(2), dz.sum(2)
    m = P * (C // G)
    s1, s2 = ((q * gamma[:, None, :]).view(K, N, G, C // G).sum(3) / m for q in (B, A))
    t = (dz * gamma[:, None, None, :]).view(K, N, P, G, C // G)
    t = t - s1[:, :, None, :, None] - xh.view(t.shape) * s2[:, :, None, :, None]
    return (t * rstd[:, :, None, :, None]).view(K, N, P, C), A.sum(1), B.sum(1)


def _plain_gn(s):
    c, x = s["case"], s["x"].float()
    if c["op"] == "gn_fwd":
        mean, rstd = _gn_stats(x, c["G"])
        y = _act(_gn_z(x, mean, rstd, s["gamma"], s["beta"])[1], c["act"])
        return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}
    dx, dg, db = _gn_backward(s["dy"].float(), x, s["mean"], s["rstd"], s["gamma"], s["beta"],
                              c["act"])
    C, pad = c["C"], s["gpar"].shape[1] // 2
    s["gpar"][:, :C], s["gpar"][:, pad:pad + C] = dg, db
    return {"dx": dx.to(s["x"].dtype), "g": s["gpar"]}


# ------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    if c["op"].startswith("gn"):
        return _own_gn(s) if own else _plain_gn(s)
    if c["op"] == "step":
        if own:
            S = s["S"]
            S.saef_round_end_clipped(s["layout"], s["t"], 0, c["K"], LR, c["mu"], S.MODE_DC,
                                     s["max_norm"], s["norms"], s["g"], s["m"], s["e"],
                                     s["e_srv"], s["x"], s["signs"], s["scales"],
                                     s["srv_signs"], s["srv_scales"])
        else:
            _plain_step(s)
        s["t"] += 1
        return _step_out(s)
    max_norm = s["max_norm"]
    if c["op"] == "clip" and c["out"] == "same":
        # the bound tightens from step to step, so that gradients already clipped are
        # clipped again
        s["max_norm"] *= 0.999
    if not own:
        return _plain_norm(s) if c["op"] == "norm" else _plain_clip(s, max_norm)
    S = s["S"]
    S.saef_grad_norm(s["grads"], s["norms"], tensor_norms=s["tnorms"],
                     norm_type=2 if c["p"] == "2" else math.inf)
    out = {"norms": s["norms"]}
    if c["per_tensor"]:
        out["tensor_norms"] = s["tnorms"]
    if c["op"] == "clip":
        S.saef_clip(s["grads"], max_norm, s["norms"], out=s.get("rows"))
        out["clipped"] = (s["rows"] if c["out"] == "rows" else s["g"] if c["src"] == "rows"
                          else s["bucket"])
    return out


def _own_gn(s):
    S = s["S"]
    if s["case"]["op"] == "gn_fwd":
        S.saef_group_norm_forward(s["plan"], s["x"], s["gamma"], s["beta"], s["out"], s["mean"],
                                  s["rstd"])
        return {"y": s["out"], "mean": s["mean"], "rstd": s["rstd"]}
    C, pad = s["case"]["C"], s["gpar"].shape[1] // 2
    S.saef_group_norm_backward(s["plan"], s["dy"], s["x"], s["gamma"], s["beta"], s["mean"],
                               s["rstd"], s["out"], s["gpar"][:, :C], s["gpar"][:, pad:pad + C])
    return {"dx": s["out"], "g": s["gpar"]}


# ------------------------------------------------------------------ what a pass needs

def work(case):
    """Every input read once and every output written once."""
    K = case["K"]
    if case["op"].startswith("gn"):
        n = K * case["N"] * case["P"] * case["C"]
        es = 4 if case["dtype"] == "f32" else 2
        small = 2 * 4 * K * case["N"] * case["G"] + 2 * 4 * K * case["C"]
        if case["op"] == "gn_fwd":
            return {"bytes": 2 * es * n + small, "flops": 8.0 * n}
        return {"bytes": 3 * es * n + small + 2 * 4 * K * case["C"], "flops": 18.0 * n}
    lay = _Layout(case)
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "step":
        # g, e, old words in; e, words out (and momentum both ways); the server's error,
        # weights and words in and out
        b = (12 + 2 / 8 + (8 if case["mu"] else 0)) * K + 16 + 2 / 8
        return {"bytes": b * lay.d + 8 * (K + 1) * lay.L, "flops": (5.0 * K + 6) * lay.d}
    b = es * K * lay.d + 4 * K + (4 * K * lay.L if case["per_tensor"] else 0)
    if case["op"] == "norm":
        return {"bytes": b, "flops": 2.0 * K * lay.d}
    b += (4 if case["out"] == "rows" else es) * K * lay.d
    return {"bytes": b, "flops": 3.0 * K * lay.d}


# ------------------------------------------------------------------ 64-bit results

def exact(case, seed):
    if case["op"].startswith("gn"):
        return _exact_gn(case, seed)
    return _exact_step(case, seed) if case["op"] == "step" else _exact_clip(case, seed)


def _exact_clip(case, seed):
    s = _prepare_plain(case, seed)
    lay, K = s["lay"], case["K"]
    norms, tnorms, rows = [], [], []
    for k in range(K):
        parts = lay.slices(s["g"][k]) if case["src"] == "rows" else s["list"][k]
        if case["p"] == "2":
            q = torch.stack([torch.dot(v.double(), v.double()) for v in parts])
            norms.append(math.sqrt(math.fsum(q.tolist())))
            tnorms.append(q.sqrt())
        else:
            q = torch.stack([torch.maximum(v.max(), -v.min()).double() for v in parts])
            norms.append(float(q.max()))
            tnorms.append(q)
        if case["op"] == "clip":
            f = min(1.0, s["max_norm"] / (norms[-1] + TINY))
            row = torch.zeros(lay.d_pad, dtype=torch.float64, device="cuda")
            for o, n, v in zip(lay.off, lay.n, parts):
                row[o:o + n] = v.double() * f
            rows.append(row)
    out = {"norms": torch.tensor(norms, dtype=torch.float64, device="cuda")}
    if case["per_tensor"]:
        out["tensor_norms"] = torch.stack(tnorms)
    if case["op"] == "clip":
        if case["out"] == "same" and case["src"] == "list":
            rows = [torch.cat(lay.slices(r)) for r in rows]
        out["clipped"] = torch.stack(rows)
    return out


def _prepare_plain(case, seed):
    """prepare's data without the framework's handles."""
    global own
    was, own = own, False
    try:
        return _prepare_grad(case, seed)
    finally:
        own = was


def _exact_step(case, seed):
    """Algorithm 1's second half in 64 bits.  Signs of sums that rounding decides are no
    computed numbers, so the words have no value here; the scales hardly feel them, and the server's
    error and weights are taken from the message's 32-bit values."""
    s = _prepare_plain(case, seed)
    lay, K = s["lay"], case["K"]
    lr, mu = (float(torch.tensor(v, dtype=torch.float32)) for v in (LR, case["mu"]))
    max_norm = float(torch.tensor(s["max_norm"], dtype=torch.float32))
    e, m, scales = [], [], []
    total = torch.zeros(lay.d_pad, dtype=torch.float64, device="cuda")
    for k in range(K):
        f = min(1.0, max_norm / (float(s["norms"][k]) + TINY))
        step = s["g"][k].double() * f
        if case["mu"]:
            step = step + mu * s["m"][k].double()
            m.append(step)
        v = s["e"][k].double() - _decode(lay, s["signs"][k], s["scales"][k].double()) + lr * step
        e.append(v)
        scales.append(torch.stack([p.abs().mean() for p in lay.slices(v)]))
        spread = lay.per_element(scales[-1])
        total += torch.where(v >= 0, spread, -spread)
    old = _decode(lay, s["srv_signs"], s["srv_scales"].double())
    es = s["e_srv"].double() - old + total / K
    out = {"e": torch.stack(e), "signs": None, "scales": torch.stack(scales),
           # one worker's undecided sign moves these by a whole step
           "e_srv": None, "srv_signs": None,
           "srv_scales": torch.stack([p.abs().mean() for p in lay.slices(es)]),
           "x": s["x"].double() - old}
    if m:
        out["m"] = torch.stack(m)
    return out


def _exact_gn(case, seed):
    x, par, gamma, beta, dy = _gn_inputs(case, seed)
    K, N, P, C, G = (case[k] for k in ("K", "N", "P", "C", "G"))
    Cg, pad = C // G, par.shape[1] // 2
    if case["op"] == "gn_bwd":
        mean, rstd = (v.double() for v in _gn_saved(case, x, gamma, beta, dy))
    ys, means, rstds, gpar = [], [], [], torch.zeros_like(par, dtype=torch.float64)
    for k in range(K):
        # group by group: (N, P Cg) at a time
        v = x[k].double().view(N, P, G, Cg)
        w, b = (q[k].double().view(G, Cg) for q in (gamma, beta))
        if case["op"] == "gn_fwd":
            mu = v.sum((1, 3)) / (P * Cg)
            r = (((v - mu[:, None, :, None]) ** 2).sum((1, 3)) / (P * Cg) + EPS) ** -0.5
            means.append(mu)
            rstds.append(r)
        else:
            mu, r = mean[k], rstd[k]
        h = (v - mu[:, None, :, None]) * r[:, None, :, None]
        z = h * w + b
        if case["op"] == "gn_fwd":
            y = z.clamp(min=0) if case["act"] == "relu" else z
            y = z * torch.sigmoid(z) if case["act"] == "silu" else y
            ys.append(y.view(N, P, C))
            continue
        d = dy[k].double().view(N, P, G, Cg)
        if case["act"] == "relu":
            d = torch.where(z > 0, d, 0.0)
        elif case["act"] == "silu":
            sg = torch.sigmoid(z)
            d = d * (sg + z * sg * (1 - sg))
        gpar[k, :C] = (d * h).sum((0, 1)).view(C)
        gpar[k, pad:pad + C] = d.sum((0, 1)).view(C)
        d = d * w
        d1 = d.sum((1, 3), keepdim=True) / (P * Cg)
        d2 = (d * h).sum((1, 3), keepdim=True) / (P * Cg)
        ys.append(((d - d1 - h * d2) * r[:, None, :, None]).view(N, P, C))
    if case["op"] == "gn_fwd":
        return {"y": torch.stack(ys), "mean": torch.stack(means), "rstd": torch.stack(rstds)}
    return {"dx": torch.stack(ys), "g": gpar}
