"""Projections of real-valued activations: scales that are not finite, groups without rows, many groups, forms of tiles and parts, rows of odd strides."""
import pytest
import torch

from gpu_util import Guarded
from paper_2110_09195_amd import binding as B
from test_gpu_linear import Layer, normal, offsets_of

pytestmark = pytest.mark.gpu


# channels, rows of the other group: tiles of 128 x 128 whole, in parts, of 256 x 256
@pytest.mark.parametrize("ci, co, n", [(72, 40, 30), (136, 264, 2100), (4104, 4104, 300)])
@pytest.mark.parametrize("kept", [False, True])
def test_gradients_of_a_group_without_rows_are_zero_whatever_its_scales(ci, co, n, kept):
    print("case", ci, co, n, kept, flush=True)
    L = Layer(1, 2, ci, co, 16, "bf16")
    alpha = L.alpha.clone()
    alpha[0, 0], alpha[0, 1], alpha[0, 2:] = float("nan"), float("inf"), float("-inf")
    weights = B.snn_linear_prepare(L.desc, L.codebook, L.idx, alpha)
    x, dy, off = L.rows(1, n, ci), L.rows(2, n, co), offsets_of([0, n])
    arg = B.snn_checkpoint_store(x) if kept else x
    (dw, da), (want, want_a) = (B.snn_linear_weight_grad(L.desc, arg, dy, w, offsets=off) for w in (weights, L.weights))
    assert torch.equal(dw, want) and torch.equal(da, want_a) and not bool(dw[0].any()) and not bool(da[0].any()) and bool(dw[1].any())
    none = [B.snn_linear_weight_grad(L.desc, x[:0], dy[:0], weights, offsets=offsets_of([0, 0]))[0]]
    assert not bool(none[0].any())


# one part of the rows, and several
@pytest.mark.parametrize("T, n", [(60, 3), (4000, 2)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_scale_that_is_not_finite_shows_in_its_own_gradients(T, n, bad):
    """dB = scale * sum dy low: where the sum is zero and the scale is infinite or NaN, that is NaN; an adapter without rows has zeros."""
    L, r = Layer(2, 1, 72, 40, 16, "bf16"), 8
    x, dy = L.rows(1, T, 72), L.rows(2, T, 40)
    dy[:, 5] = 0.0
    A, Bm = normal(3, n + 1, r, 72).to(L.dtype), normal(4, n + 1, 40, r).to(L.dtype)
    ids = (torch.arange(T, device="cuda") * n // T).int()
    scale = torch.full((n + 1,), 2.0, device="cuda")
    y, low = B.snn_adapters_forward(L.desc, x, L.weights, ids, A, Bm, scale)
    _, _, want = B.snn_adapters_backward(L.desc, x, low, dy, L.weights, ids, A, Bm, scale)
    scale[1], scale[n] = bad, bad                            # (nobody has the last)
    _, dA, dB = B.snn_adapters_backward(L.desc, x, low, dy, L.weights, ids, A, Bm, scale)
    assert bool(dB[1, 5].isnan().all()) and not bool(want[1, 5].any()) and not bool(dB[1].isfinite().any()) and not bool(dA[1].isfinite().any())
    assert torch.equal(dB[0], want[0]) and not bool(dB[n].any()) and not bool(dA[n].any())


@pytest.mark.parametrize("native", [True, False])
def test_a_single_row_of_any_view(native, monkeypatch):
    """The last token of a long sequence, a row of an odd distance: the distance of a single row does not count."""
    if not native:
        B.lib()
        monkeypatch.setattr(B, "_fast", None)
    L, r = Layer(3, 1, 4096, 72, 16, "bf16"), 8
    A, Bm, scale = normal(3, 2, r, 4096).to(L.dtype), normal(4, 2, 72, r).to(L.dtype), normal(5, 2)
    ids = torch.zeros(1, dtype=torch.int32, device="cuda")
    sequence = normal(1, 1, 300, 4096).to(L.dtype)
    odd, odd_dy = normal(2, 1, 4099).to(L.dtype), normal(6, 1, 75).to(L.dtype)
    for x, dy in ((sequence[:, -1], odd_dy[:, :72]), (odd[:, :4096], odd_dy[:, :72])):
        assert x.stride(0) > 4096 and dy.stride(0) == 75
        own, own_dy = x.clone(), dy.clone()
        assert torch.equal(B.snn_linear_forward(L.desc, x, L.weights), B.snn_linear_forward(L.desc, own, L.weights))
        assert torch.equal(B.snn_linear_input_grad(L.desc, dy, L.weights), B.snn_linear_input_grad(L.desc, own_dy, L.weights))
        kept, want = B.snn_checkpoint_store(x), B.snn_checkpoint_store(own)
        assert all(torch.equal(a, b) for a, b in zip(kept, want))
        out = torch.zeros(1, 4099, device="cuda").to(L.dtype)
        assert torch.equal(B.snn_checkpoint_restore(kept, L.dtype, x=out[:, :4096]), B.snn_checkpoint_restore(want, L.dtype))
        assert torch.equal(B.snn_linear_weight_grad(L.desc, x, dy, L.weights)[0], B.snn_linear_weight_grad(L.desc, own, own_dy, L.weights)[0])
        (y, low), (want, _) = (B.snn_adapters_forward(L.desc, v, L.weights, ids, A, Bm, scale) for v in (x, own))
        assert torch.equal(y, want)
        got, want = (B.snn_adapters_backward(L.desc, v, low, d, L.weights, ids, A, Bm, scale) for v, d in ((x, dy), (own, own_dy)))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T, groups", [(90, 64), (5000, 300), (100000, 1024)])
def test_offsets_that_go_down_and_up_again_stay_inside(T, groups):
    """Every other group claims all rows: far more tiles than there can be.  What rows get is not defined, but nothing else is written."""
    L = Layer(4, groups, 16, 24, 4, "bf16")
    x, dy = L.rows(1, T, 16), L.rows(2, T, 24)
    off = torch.tensor([0, T] * (groups // 2) + [0] * (1 + groups % 2), dtype=torch.int32, device="cuda")
    g, y = L.out(T, 24, 8)
    B.snn_linear_forward(L.desc, x, L.weights, offsets=off, y=y)
    g.check("y")
    assert bool(g.t.view(T, 32)[:, 24:].isnan().all())
    g, dx = L.out(T, 16, 8)
    B.snn_linear_input_grad(L.desc, dy, L.weights, offsets=off, dx=dx)
    g.check("dx")
    assert bool(g.t.view(T, 24)[:, 16:].isnan().all())
    g = Guarded(groups * 24 * 16, torch.float32)
    B.snn_linear_weight_grad(L.desc, x, dy, L.weights, offsets=off, dw=g.t.view(groups, 24, 16))
    g.check("dw")


# few rows, tiles
@pytest.mark.parametrize("T, ci, co", [(9, 64, 72), (400, 136, 4104), (1500, 264, 520)])
def test_values_below_the_normal_numbers_of_f16_count(T, ci, co):
    """Multiples of 2^-24, the smallest f16 value: whole numbers times it, whose sums are exact."""
    L, r, unit = Layer(6, 1, ci, co, 16, "f16"), 8, 2.0 ** -24
    L.weights = B.snn_linear_prepare(L.desc, L.codebook, L.idx, torch.ones(1, co, device="cuda").half())

    def whole(seed, *shape):
        return (normal(seed, *shape) * 3).round().clamp(-9, 9).double()
    x, dy = whole(1, T, ci), whole(2, T, co)
    tiny_x, tiny_dy = (x * unit).half(), (dy * unit).half()
    assert torch.equal(tiny_x.double(), x * unit)
    assert torch.equal(B.snn_linear_forward(L.desc, tiny_x, L.weights).double(), x @ L.w[0].t() * unit)
    assert torch.equal(B.snn_linear_input_grad(L.desc, tiny_dy, L.weights).double(), dy @ L.w[0] * unit)
    dw, _ = B.snn_linear_weight_grad(L.desc, tiny_x, dy.half(), L.weights)
    assert torch.equal(dw[0].double(), dy.t() @ x * unit)
    kept = B.snn_checkpoint_restore(B.snn_checkpoint_store(tiny_x), L.dtype)
    assert torch.equal(kept, tiny_x)
    A, Bm, one = whole(3, 1, r, ci), torch.zeros(1, co, r, dtype=torch.float64, device="cuda"), torch.ones(1, device="cuda")
    Bm[0, :, 3] = 1.0
    ids = torch.zeros(T, dtype=torch.int32, device="cuda")
    y, low = B.snn_adapters_forward(L.desc, tiny_x, L.weights, ids, A.half(), Bm.half(), one)
    assert torch.equal(low.double(), x @ A[0].t() * unit)
    assert torch.equal(y.double(), ((x @ L.w[0].t() + (x @ A[0].t())[:, 3:4]) * unit).half().double())
