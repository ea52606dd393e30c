"""Adapters' inner products enter their second products with the precision of fp32, however many rows a call has.

Whole numbers: inner products of some 20 bits meet factors of +-1 in pairs, so that all but their last bits cancel.  Every sum in any order is of
whole numbers below 2^24 (times one power of two), so results have to be those of 64 bits, rounded once; an inner product that has lost a bit shows."""
import numpy as np
import pytest
import torch

from paper_2110_09195_amd import binding as B

pytestmark = pytest.mark.gpu

# rows, C_in, C_out: many rows (tiles), many rows of ragged widths, wide outputs, wide inputs, few rows
SHAPES = [(20512, 64, 64), (20500, 72, 40), (3000, 64, 1032), (3000, 1032, 64), (304, 64, 4104), (400, 4104, 64), (200, 64, 64)]
RANKS = [8, 24, 64, 72]
# type, and the powers of two on vectors, on the matrices that make inner products, and on the factors of +-1
KINDS = [("bf16", 1.0, 1.0, 1.0)]
TYPES = {"bf16": (torch.bfloat16, B.SNN_DTYPE_BF16), "f16": (torch.float16, B.SNN_DTYPE_F16)}
N = 3


def numbers(seed, shape, C):
    """Whole numbers such that the inner product of two vectors of C of them has about 20 bits, and no more"""
    lo, hi = (8, 15) if C > 1000 else (64, 127) if C > 40 else (80, 127)
    return torch.from_numpy(np.random.default_rng(seed).integers(lo, hi + 1, shape).astype(np.float64)).cuda()


def near_pairs(seed, shape):
    """[..., 2 pairs, C]: the second of two differs from the first by 1 in one place"""
    *rest, twice, C = shape
    first = numbers(seed, (*rest, twice // 2, C), C)
    at = torch.from_numpy(np.random.default_rng(seed + 1).integers(0, C, first.shape[:-1])).cuda()[..., None]
    second = first.scatter_add(-1, at, torch.ones_like(at, dtype=torch.float64))
    return torch.stack([first, second], -2).view(shape)


def opposites(seed, shape):
    """[..., 2 pairs, C] of +-1: the second of two is the first's opposite"""
    *rest, twice, C = shape
    one = torch.from_numpy(np.random.default_rng(seed).choice([-1.0, 1.0], (*rest, twice // 2, C))).cuda()
    return torch.stack([one, -one], -2).view(shape)


def setting(T, ci, co, name):
    """A projection whose scales are zero (outputs are the adapters' share alone), and rows in runs of 16 of one adapter or none"""
    dtype, code = TYPES[name]
    desc = B.make_linear_desc(1, ci, co, 1, code)
    codes, idx = torch.zeros(1, 1, dtype=torch.int16, device="cuda"), torch.zeros(1, co, ci // 8, dtype=torch.int16, device="cuda")
    weights = B.snn_linear_prepare(desc, codes, idx, torch.zeros(1, co, device="cuda").to(dtype))
    ids = np.random.default_rng(5).integers(-1, N, T // 16 + 1).repeat(16)[:T].astype(np.int32)
    return desc, dtype, weights, torch.from_numpy(ids).cuda(), torch.ones(N, device="cuda")


def products(v, down, up, ids):
    """(up (down v_t), down v_t) of each row's adapter, in 64 bits: down [n][rank][C], up [n][C'][rank]"""
    low = torch.zeros(v.shape[0], down.shape[1], dtype=torch.float64, device="cuda")
    out = torch.zeros(v.shape[0], up.shape[1], dtype=torch.float64, device="cuda")
    for a in range(N):
        low[ids == a] = v[ids == a] @ down[a].t()
        out[ids == a] = low[ids == a] @ up[a].t()
    assert float(low.abs().amax()) >= 2 ** 18 * float(v.abs().amax() * down.abs().amax()) / 127 ** 2 / 8     # (of the size that is meant)
    return out, low


def turned(t):
    return t.transpose(1, 2).contiguous()


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("T, ci, co", SHAPES)
def test_outputs_and_gradients_of_inputs(T, ci, co, rank, kind):
    name, pv, pm, pf = KINDS[kind]
    print("case", T, ci, co, rank, name, pv, flush=True)
    desc, dtype, w, ids, one = setting(T, ci, co, name)
    x, A, Bm = pv * numbers(1, (T, ci), ci), pm * near_pairs(2, (N, rank, ci)), pf * turned(opposites(3, (N, rank, co)))
    want, low = products(x, A, Bm, ids)
    y, got = B.snn_adapters_forward(desc, x.to(dtype), w, ids, A.to(dtype), Bm.to(dtype), one)
    assert torch.equal(got.double(), low)
    assert torch.equal(y, want.to(dtype))
    dy, A, Bm = pv * numbers(4, (T, co), co), pf * opposites(5, (N, rank, ci)), pm * turned(near_pairs(6, (N, rank, co)))
    want, _ = products(dy, turned(Bm), turned(A), ids)
    dx, _, _ = B.snn_adapters_backward(desc, x.to(dtype), got, dy.to(dtype), w, ids, A.to(dtype), Bm.to(dtype), one)
    assert torch.equal(dx, want.to(dtype))


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("rank", RANKS)
@pytest.mark.parametrize("T, ci, co", SHAPES)
def test_gradients_of_adapters(T, ci, co, rank, kind):
    name, pv, pm, pf = KINDS[kind]
    print("case", T, ci, co, rank, name, pv, flush=True)
    desc, dtype, w, ids, one = setting(T, ci, co, name)
    members = [(a, ids == a) for a in range(N)]

    def backward(x, low, dy, A, Bm, kept):
        x = x.to(dtype)
        return B.snn_adapters_backward(desc, B.snn_checkpoint_store(x) if kept else x, low.float(), dy.to(dtype), w, ids, A.to(dtype), Bm.to(dtype), one)

    # dA: rows in opposite pairs, inner products of the gradients in near ones
    x, dy, A, Bm = pf * opposites(1, (T, ci)), pv * near_pairs(2, (T, co)), pm * numbers(3, (N, rank, ci), ci), pm * numbers(4, (N, co, rank), co)
    _, dlow = products(dy, turned(Bm), turned(A), ids)
    want = torch.stack([dlow[rows].t() @ x[rows] for _, rows in members])
    for kept in (False, True):
        _, dA, _ = backward(x, torch.zeros(T, rank, device="cuda"), dy, A, Bm, kept)
        assert torch.equal(dA, want.to(dtype)), kept
    # dB: the other way round
    x, dy = pv * near_pairs(5, (T, ci)), pf * opposites(6, (T, co))
    _, low = products(x, A, Bm, ids)
    want = torch.stack([dy[rows].t() @ low[rows] for _, rows in members])
    _, _, dB = backward(x, low, dy, A, Bm, False)
    assert torch.equal(dB, want.to(dtype))
