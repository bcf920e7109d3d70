"""A small residual network trained by K workers with clipped, compressed gradients.

    python -m paper_2008_05823_amd.example_training [--steps 200] [--workers 8]

Each iteration is one of Algorithm 1: ``saef_round_begin`` writes the K evaluation
points xh; the network runs at all of them at once, its group norms reading their
parameters from the rows of xh and writing those gradients into the gradient rows g;
``saef_grad_norm`` takes each worker's norm and ``saef_round_end_clipped`` clips,
compresses, aggregates and updates.  The images are synthetic, labelled by a fixed
random linear map of their mean pixel.

The network, on images of P pixels by 12 channels, channels last:
    a = silu(group_norm(images W1));  b = a + relu(group_norm(a W2))
    logits = mean over pixels of b, times W3, plus b3
"""
from __future__ import annotations

import argparse

import torch

from . import saef as S

IN, WIDTH, CLASSES, GROUPS = 12, 32, 10, 8


class Network:
    """Parameters as slices of a flat layout, for K workers' rows at once."""

    shapes = (("w1", (IN, WIDTH)), ("gamma1", (WIDTH,)), ("beta1", (WIDTH,)),
              ("w2", (WIDTH, WIDTH)), ("gamma2", (WIDTH,)), ("beta2", (WIDTH,)),
              ("w3", (WIDTH, CLASSES)), ("b3", (CLASSES,)))

    def __init__(self, K: int, N: int, P: int):
        self.K, self.N, self.P = K, N, P
        self.at, at = {}, 0
        for name, shape in self.shapes:
            n = torch.Size(shape).numel()
            self.at[name] = (at, n, shape)
            at += (n + 63) // 64 * 64
        self.d_pad = at
        self.layout = S.Layout([o for o, _, _ in self.at.values()],
                               [n for _, n, _ in self.at.values()], at, K)
        norm = dict(K=K, N=N, P=P, C=WIDTH, G=GROUPS, dtype=torch.float32)
        self.norm1 = S.GroupNorm(act=S.ACT_SILU, **norm)
        self.norm2 = S.GroupNorm(act=S.ACT_RELU, **norm)

        def features():
            return torch.empty((K, N, P, WIDTH), device="cuda")

        def stats():
            return torch.empty((K, N, GROUPS), device="cuda")
        self.f = {k: features() for k in ("u1", "a", "u2", "r", "d", "e")}
        self.s = {k: stats() for k in ("mean1", "rstd1", "mean2", "rstd2")}

    def part(self, rows, name):
        """Parameter `name` of every worker: a view of rows (K, d_pad)."""
        o, n, shape = self.at[name]
        return rows[:, o:o + n].view(rows.shape[0], *shape)

    def initial(self, seed: int):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        x = torch.zeros((1, self.d_pad), device="cuda")
        for name, (o, n, shape) in self.at.items():
            if name.startswith("w"):
                x[0, o:o + n] = torch.randn(n, generator=gen, device="cuda") / shape[0] ** 0.5
            elif name.startswith("gamma"):
                x[0, o:o + n] = 1.0
        return x[0]

    def gradient(self, xh, images, labels, g):
        """Writes the K gradients at the rows of xh into the rows of g; the mean loss."""
        K, N, P, f, s = self.K, self.N, self.P, self.f, self.s

        def p(name):
            return self.part(xh, name)

        def flat(v):
            return v.view(K, N * P, -1)
        torch.bmm(flat(images), p("w1"), out=flat(f["u1"]))
        S.saef_group_norm_forward(self.norm1, f["u1"], p("gamma1"), p("beta1"), f["a"],
                                  s["mean1"], s["rstd1"])
        torch.bmm(flat(f["a"]), p("w2"), out=flat(f["u2"]))
        S.saef_group_norm_forward(self.norm2, f["u2"], p("gamma2"), p("beta2"), f["r"],
                                  s["mean2"], s["rstd2"])
        pooled = (f["a"] + f["r"]).mean(2)                       # (K, N, WIDTH)
        logits = torch.bmm(pooled, p("w3")) + p("b3")[:, None]
        logp = torch.log_softmax(logits, -1)
        loss = -logp.gather(-1, labels[..., None]).mean()

        # backward
        dl = logp.exp()
        dl.scatter_add_(-1, labels[..., None], torch.full_like(dl[..., :1], -1.0))
        dl /= N
        self.part(g, "w3").copy_(torch.bmm(pooled.transpose(1, 2), dl))
        self.part(g, "b3").copy_(dl.sum(1))
        db = torch.bmm(dl, p("w3").transpose(1, 2).contiguous()) / P  # of every pixel
        db = db[:, :, None].expand(K, N, P, WIDTH).contiguous()
        S.saef_group_norm_backward(self.norm2, db, f["u2"], p("gamma2"), p("beta2"), s["mean2"],
                                   s["rstd2"], f["d"], self.part(g, "gamma2"),
                                   self.part(g, "beta2"))
        self.part(g, "w2").copy_(torch.bmm(flat(f["a"]).transpose(1, 2), flat(f["d"])))
        da = flat(db) + torch.bmm(flat(f["d"]), p("w2").transpose(1, 2).contiguous())
        S.saef_group_norm_backward(self.norm1, da.view(K, N, P, WIDTH), f["u1"], p("gamma1"),
                                   p("beta1"), s["mean1"], s["rstd1"], f["e"],
                                   self.part(g, "gamma1"), self.part(g, "beta1"))
        self.part(g, "w1").copy_(torch.bmm(flat(images).transpose(1, 2), flat(f["e"])))
        return loss


def batch(net: Network, seed: int):
    """K workers' images and labels."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    teacher = torch.randn((IN, CLASSES), generator=gen, device="cuda")
    gen.manual_seed(seed)
    images = torch.randn((net.K, net.N, net.P, IN), generator=gen, device="cuda")
    images += 2.0 * torch.randn((net.K, net.N, 1, IN), generator=gen, device="cuda")
    return images, (images.mean(2) @ teacher).argmax(-1)


def train(K=8, N=16, P=64, steps=200, lr=0.3, max_norm=1.0, period=20, seed=0, report=None):
    """Trains and returns the losses of the steps (a device tensor)."""
    net = Network(K, N, P)
    d, W = net.d_pad, net.d_pad // 64
    x = net.initial(seed)
    e, xh, g = (torch.zeros((K, d), device="cuda") for _ in range(3))
    e_srv = torch.zeros(d, device="cuda")
    L = len(net.at)
    signs, scales = torch.zeros((K, W), dtype=torch.int64, device="cuda"), torch.zeros(
        (K, L), device="cuda")
    srv = torch.zeros(W, dtype=torch.int64, device="cuda"), torch.zeros(L, device="cuda")
    grads, norms = S.Grads(net.layout, g), torch.zeros(K, device="cuda")
    losses = torch.zeros(steps, device="cuda")
    for t in range(steps):
        S.saef_round_begin(net.layout, t, period, K, S.MODE_DC, S.VARIANT_SAEF, e, e_srv, x, xh,
                           signs, scales, *srv)
        losses[t] = net.gradient(xh, *batch(net, 1000 + t), g)
        S.saef_grad_norm(grads, norms)
        S.saef_round_end_clipped(net.layout, t, period, K, lr, 0.0, S.MODE_DC, max_norm, norms, g,
                                 None, e, e_srv, x, signs, scales, *srv)
        if report and (t + 1) % report == 0:
            print(f"step {t + 1:4d}  loss {float(losses[t]):.4f}  norms "
                  f"{float(norms.min()):.3f} to {float(norms.max()):.3f}", flush=True)
    if S.saef_status(net.layout) != S.OK:
        raise RuntimeError("values left the range of the exact sums")
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--max-norm", type=float, default=1.0)
    a = ap.parse_args()
    losses = train(K=a.workers, steps=a.steps, max_norm=a.max_norm, report=max(1, a.steps // 10))
    print(f"mean loss of the first and last tenth: {float(losses[:a.steps // 10 + 1].mean()):.4f} "
          f"{float(losses[-(a.steps // 10 + 1):].mean()):.4f}")


if __name__ == "__main__":
    main()
