"""Norms of the .grad tensors of automatic differentiation, kept and allocated anew."""
import pytest
import torch

from paper_2008_05823_amd import workloads as W

pytestmark = pytest.mark.gpu

SIZES = [4000, 70, 5]


def test_grad_tensors_kept_and_new():
    """A Grads reads the tensors it was made of.  zero_grad(set_to_none=False) leaves them in
    place, so it goes on; after set_to_none=True there are other tensors, which need another Grads,
    while the first still stands for the old ones.  Whole numbers: the norms are exact."""
    from paper_2008_05823_amd import saef as S
    off, n, d_pad = W.custom(SIZES, K=1).layout()
    lay = S.Layout(off, n, d_pad, 1)
    params = [torch.zeros(m, device="cuda", requires_grad=True) for m in SIZES]
    opt = torch.optim.SGD(params, lr=0.1)
    norms = torch.zeros(1, device="cuda")

    def backward(c):
        sum((c * p).sum() for p in params).backward()

    def norm(grads):
        S.saef_grad_norm(grads, norms)
        return float(norms)

    def want(c):
        return float(torch.tensor(c * c * sum(SIZES), dtype=torch.float64).sqrt().float())
    backward(3.0)
    kept = S.Grads(lay, [[p.grad for p in params]])
    assert norm(kept) == want(3.0)
    opt.zero_grad(set_to_none=False)
    backward(4.0)
    assert norm(kept) == want(4.0)
    opt.zero_grad(set_to_none=True)
    backward(5.0)
    new = S.Grads(lay, [[p.grad for p in params]])
    assert norm(new) == want(5.0)
    assert norm(kept) == want(4.0)
    S.saef_clip(new, 1.0, norms.fill_(want(5.0)))  # in place, in autograd's own tensors
    f = float(torch.tensor(1.0) / (torch.tensor(want(5.0)) + torch.tensor(1e-6)))
    for p in params:
        assert bool((p.grad == torch.tensor(5.0 * f, device="cuda")).all())
