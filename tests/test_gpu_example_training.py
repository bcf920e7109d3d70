"""The training example: its gradient against automatic differentiation in 64 bits, and
that it learns under clipping and compression."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _loss(net, rows, images, labels):
    """The example's network in elementary operations, one worker's row at a time."""
    from paper_2008_05823_amd import example_training as X

    def norm(v, gamma, beta):
        q = v.view(net.N, net.P, X.GROUPS, -1)
        m = q.mean((1, 3), keepdim=True)
        var = ((q - m) ** 2).mean((1, 3), keepdim=True)
        return ((q - m) / torch.sqrt(var + 1e-5)).view(v.shape) * gamma + beta
    total = 0.0
    for k in range(net.K):
        def p(name):
            o, n, shape = net.at[name]
            return rows[k, o:o + n].view(shape)
        z = norm(images[k] @ p("w1"), p("gamma1"), p("beta1"))
        a = z / (1 + torch.exp(-z))
        b = a + norm(a @ p("w2"), p("gamma2"), p("beta2")).clamp(min=0)
        logits = b.mean(1) @ p("w3") + p("b3")
        total = total - torch.log_softmax(logits, -1).gather(-1, labels[k][:, None]).mean()
    return total


def test_gradient():
    """A chain of some ten fp32 operations with sums of up to 1024 terms: 1e-4 of the
    gradient's largest entry is 100 times their expected rounding."""
    from paper_2008_05823_amd import example_training as X
    net = X.Network(3, 4, 37)
    images, labels = X.batch(net, 5)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    xh = net.initial(0)[None] + 0.1 * torch.randn((3, net.d_pad), generator=gen, device="cuda")
    g = torch.zeros_like(xh)
    loss = net.gradient(xh, images, labels, g)
    rows = xh.double().cpu().requires_grad_()
    want = _loss(net, rows, images.double().cpu(), labels.cpu())
    want.backward()
    assert abs(float(loss) - float(want.detach()) / 3) < 1e-5
    diff = (g.cpu().double() - rows.grad).abs().max()
    assert float(diff) <= 1e-4 * float(rows.grad.abs().max())


def test_it_learns():
    from paper_2008_05823_amd import example_training as X
    losses = X.train(K=4, steps=150)
    assert float(losses[-15:].mean()) < 0.5 * float(losses[:15].mean())
