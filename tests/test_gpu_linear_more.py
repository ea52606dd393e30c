"""The checks of test_gpu_linear.py at more sizes: more than 64 groups (which are looked over 64 at a time), weights' gradients in four parts, input gradients
in tiles beside adapters of more than 64, and more rows than the kernels of few rows take, each with an adapter of its own."""
import pytest

import test_gpu_linear as T

pytestmark = pytest.mark.gpu

SHAPES = [
    # few rows a group, and tiles
    ([3] * 65, 72, 40, 16, 0), ([k % 7 for k in range(128)], 136, 264, 32, 8), ([0] * 63 + [5] + [0] * 64 + [9, 0], 64, 72, 4, 0),
    ([40] * 256, 136, 520, 8, 0), ([k * k % 150 for k in range(129)], 200, 776, 64, 8), ([k % 3 for k in range(1024)], 40, 24, 2, 0),
    ([0] * 700 + [300, 0, 1, 2000] + [0] * 320, 72, 520, 16, 0),
    # weights' gradients in four parts
    ([1100], 136, 1416, 32, 0), ([1050, 1060], 136, 264, 16, 8),
]

ADAPTED = [
    (3001, 4104, 136, 3, 72, "wild"), (3001, 4104, 136, 2, 128, "runs"), (2500, 2904, 2056, 4, 104, "sorted"),
    (256, 1032, 4104, 64, 16, "each"), (512, 4104, 520, 64, 64, "each"), (131, 4104, 4104, 100, 72, "each"),
]


@pytest.mark.parametrize("dtype", sorted(T.DTYPES))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_groups(shape, dtype, monkeypatch):
    monkeypatch.setattr(T, "SHAPES", SHAPES)
    T.test_forward_and_input_grad(shape, dtype)
    for kept in (False, True):
        T.test_weight_grad(shape, dtype, kept)


@pytest.mark.parametrize("dtype", sorted(T.DTYPES))
@pytest.mark.parametrize("case", range(len(ADAPTED)))
def test_adapters(case, dtype, monkeypatch):
    monkeypatch.setattr(T, "ADAPTED", ADAPTED)
    T.test_adapters(case, dtype)
