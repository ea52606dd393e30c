"""The layers over tokens: their gradients against automatic differentiation in 64 bits, training, serving."""
import pytest
import torch

from paper_2110_09195_amd import binding as B
from paper_2110_09195_amd import token_layers as TL

pytestmark = pytest.mark.gpu


def _near(got, want, unit, name):
    """Sums of products of 16-bit values, each rounded once to `unit`: a norm's error of at most that unit (and 32-bit sums below it)"""
    err = (got.double() - want).norm() / want.norm()
    assert float(err) <= unit + 1e-5, (name, float(err))


@pytest.mark.parametrize("dtype, unit", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)])
def test_gradients_of_experts(dtype, unit):
    g = torch.Generator(device="cuda").manual_seed(1)
    n, c_in, c_out, K, rows = 3, 72, 40, 16, 90
    cb = TL._random_codebook(n, K, g)
    w = torch.randn(n, c_out, c_in, generator=g, device="cuda", requires_grad=True)
    alpha = (0.5 + torch.rand(n, c_out, generator=g, device="cuda")).to(dtype).float().requires_grad_()
    order, offsets = TL.by_expert(torch.randint(0, n, (rows,), generator=g, device="cuda"), n)
    x = torch.randn(rows, c_in, generator=g, device="cuda").to(dtype)[order].requires_grad_()
    dy = torch.randn(rows, c_out, generator=g, device="cuda").to(dtype)
    for keep in (False, True):
        x.grad = w.grad = alpha.grad = None
        y = TL.experts(x, w, alpha, cb, offsets, keep)
        y.backward(dy)
        bits = ((cb.int()[:, :, None] >> torch.arange(7, -1, -1, device="cuda")) & 1).double() * 2 - 1          # [n][K][8]
        scores = torch.einsum("govj,gkj->govk", w.detach().double().view(n, c_out, -1, 8), bits)
        W = torch.stack([bits[k][scores[k].argmax(-1)].view(c_out, c_in) for k in range(n)]).requires_grad_()
        xd, ad = x.detach().double().requires_grad_(), alpha.detach().double().requires_grad_()
        kept = B.snn_checkpoint_restore(B.snn_checkpoint_store(x.detach()), dtype).double() if keep else xd.detach()
        expert = torch.bucketize(torch.arange(rows, device="cuda"), offsets[1:].long(), right=True)
        out = torch.cat([(xd[expert == k] @ W[k].t()) * ad[k] for k in range(n)])
        out.backward(dy.double())
        _near(y.detach(), out.detach(), unit, "y")
        _near(x.grad, xd.grad, unit, "dx")
        W.grad = ad.grad = None
        torch.cat([(kept[expert == k] @ W[k].t()) * ad[k] for k in range(n)]).backward(dy.double())
        _near(w.grad, W.grad, 0.0, "dw")
        _near(alpha.grad, ad.grad, 0.0, "dalpha")


@pytest.mark.parametrize("dtype, unit", [(torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)])
def test_gradients_of_adapters(dtype, unit):
    g = torch.Generator(device="cuda").manual_seed(2)
    _, (desc, weights, A, Bm, scale) = TL.train_adapters(steps=0, rows=10, n=4, rank=8, c_in=136, c_out=72, dtype=dtype)
    Bm = torch.randn(Bm.shape, generator=g, device="cuda").to(dtype)
    A, Bm = A.float().requires_grad_(), Bm.float().requires_grad_()
    rows, eye = 50, torch.eye(136, device="cuda").to(dtype)
    W = B.snn_linear_forward(desc, eye, weights).double()                     # [C_in][C_out], alpha in it
    x = torch.randn(rows, 136, generator=g, device="cuda").to(dtype).requires_grad_()
    dy = torch.randn(rows, 72, generator=g, device="cuda").to(dtype)
    adapter = torch.randint(-1, 4, (rows,), generator=g, device="cuda").int()
    some = adapter >= 0
    for keep in (False, True):
        x.grad = A.grad = Bm.grad = None
        y = TL.adapted(x, A, Bm, scale, adapter, desc, weights, keep)
        y.backward(dy)
        xd, Ad, Bd = (t.detach().double().requires_grad_() for t in (x, A, Bm))
        k = adapter.clamp(min=0).long()
        low = lambda rows: (Ad[k] @ rows[:, :, None])                         # [rows][rank][1]
        share = lambda z: torch.where(some[:, None], scale.double()[k][:, None] * (Bd[k] @ z)[:, :, 0], torch.zeros(1, dtype=torch.double, device="cuda"))
        out = xd @ W + share(low(xd))
        out.backward(dy.double())
        _near(y.detach(), out.detach(), unit, "y")
        _near(x.grad, xd.grad, unit, "dx")
        _near(Bm.grad, Bd.grad, unit, "dB")
        if keep:
            kept, Ad.grad = B.snn_checkpoint_restore(B.snn_checkpoint_store(x.detach()), dtype).double(), None
            share(low(kept)).backward(dy.double())
        _near(A.grad, Ad.grad, unit, "dA")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_training_learns(dtype):
    losses = TL.train_experts(steps=40, rows=600, n=3, c_in=128, c_out=96, dtype=dtype)
    assert losses[-1] < 0.5 * losses[0]
    losses, _ = TL.train_adapters(steps=40, rows=600, n=3, c_in=128, c_out=96, dtype=dtype)
    assert losses[-1] < 0.5 * losses[0]


def test_serving_gives_what_one_call_gives():
    _, served = TL.train_adapters(steps=3, c_in=256, c_out=136)
    x = torch.randn(5, 20, 256, device="cuda").bfloat16()
    adapter = torch.arange(20, dtype=torch.int32, device="cuda") % 8 - 1
    y = TL.serve(served, x, adapter)
    whole, _ = B.snn_adapters_forward(served[0], x.flatten(0, 1), served[1], adapter.repeat(5), *served[2:])
    # (sums in another order, rounded to 8 bits each: one unit in the last place of values below 16 at most)
    assert float((y.flatten(0, 1).float() - whole.float()).abs().max()) <= 16 * 2.0 ** -8


def test_the_command_runs(capsys):
    TL.main()
    assert "served" in capsys.readouterr().out
