"""The example's autograd functions take upstream gradients as torch hands them over: expanded (a sum's), transposed, or none at all."""
import pytest

from test_gpu_delta_block import example  # noqa: F401

pytestmark = pytest.mark.gpu


def test_sums_and_transposes(example):  # noqa: F811
    import torch
    gen = torch.Generator().manual_seed(1)
    inputs = [torch.randn(s, generator=gen).cuda().requires_grad_() for s in ((2, 20, 1, 16), (2, 20, 1, 16), (2, 20, 2, 24), (2, 20, 2), (2, 20, 2))]
    weights = torch.randn(2, 2, 24, 20, generator=gen).cuda()
    q, k, v, a, b = inputs

    def run(loss):
        o = example.gated_delta(q, k / 4, v, -a.square(), torch.sigmoid(b))
        return torch.autograd.grad(loss(o), inputs)

    for loss, same in ((lambda o: o.sum(), lambda o: (o * torch.ones_like(o)).sum()),
                       (lambda o: (o.permute(0, 2, 3, 1) * weights).sum(), lambda o: (o * weights.permute(0, 3, 1, 2).contiguous()).sum())):
        for x, y in zip(run(loss), run(same)):
            assert torch.equal(x, y)


def test_norms(example):  # noqa: F811
    import torch
    gen = torch.Generator().manual_seed(2)
    x, r = (torch.randn(6, 40, generator=gen).cuda().requires_grad_() for _ in range(2))
    w = torch.ones(40, device="cuda", requires_grad=True)
    h, y = example.block_norm(x, post=w, residual=r, pre=w)
    one = torch.autograd.grad(h.sum() + y.t().sum(), (x, r, w))
    h, y = example.block_norm(x, post=w, residual=r, pre=w)
    two = torch.autograd.grad((h * torch.ones_like(h)).sum() + (y * torch.ones_like(y)).sum(), (x, r, w))
    assert all(torch.equal(a, b) for a, b in zip(one, two))
