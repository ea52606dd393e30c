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
