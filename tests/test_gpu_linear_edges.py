"""Projections of real-valued activations: scales that are not finite, groups without rows, many groups, forms of tiles and parts, rows of odd strides."""
import pytest
import torch

from paper_2110_09195_amd import binding as B
from test_gpu_linear import Layer, offsets_of

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
