"""The differentiable layers over tokens: rows of no expert, and what they refuse."""
import pytest
import torch

from paper_2110_09195_amd import token_layers as TL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [50, 1500])
def test_rows_of_no_expert_have_zeros(rows):
    g = torch.Generator(device="cuda").manual_seed(1)
    n, c_in, c_out = 3, 72, 40
    cb = TL._random_codebook(n, 16, g)
    w, alpha = torch.randn(n, c_out, c_in, generator=g, device="cuda"), torch.ones(n, c_out, device="cuda")
    x = torch.randn(rows, c_in, generator=g, device="cuda").bfloat16().requires_grad_()
    offsets = torch.tensor([7, 20, 20, rows - 9], dtype=torch.int32, device="cuda")
    for _ in range(3):
        junk = torch.full((rows * 128,), float("nan"), device="cuda")         # (what the allocator gives next is not zeros by chance)
        del junk
        x.grad = None
        y = TL.experts(x, w, alpha, cb, offsets)
        y.backward(torch.ones_like(y))
        for t in (y.detach(), x.grad):
            assert not bool(t[:7].any()) and not bool(t[rows - 9:].any()) and bool(t[7:rows - 9].isfinite().all()) and bool(t[7:rows - 9].any(1).all())


def _adapted(**change):
    _, (desc, weights, A, Bm, scale) = TL.train_adapters(steps=0, rows=10, n=4, rank=8, c_in=136, c_out=72)
    a = dict(x=torch.randn(20, 136, device="cuda").bfloat16().requires_grad_(), A=A.float().requires_grad_(), Bm=Bm.float().requires_grad_(), scale=scale,
             adapter=torch.arange(20, dtype=torch.int32, device="cuda") % 4, desc=desc, weights=weights)
    a.update(change)
    return TL.adapted(**a), a


def test_a_second_derivative_is_refused():
    y, a = _adapted()
    grad, = torch.autograd.grad(y.float().square().sum(), a["x"], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        grad.float().square().sum().backward()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(20, 72, device="cuda").bfloat16().requires_grad_()
    w = torch.randn(1, 40, 72, device="cuda", requires_grad=True)
    y = TL.experts(x, w, torch.ones(1, 40, device="cuda"), TL._random_codebook(1, 16, g), torch.tensor([0, 20], dtype=torch.int32, device="cuda"))
    grad, = torch.autograd.grad(y.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        grad.float().square().sum().backward()


def test_a_scale_that_asks_for_a_gradient_is_refused():
    with pytest.raises(ValueError, match="scale has no gradient"):
        _adapted(scale=torch.full((4,), 2.0, device="cuda", requires_grad=True))
