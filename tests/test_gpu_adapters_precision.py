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
KINDS = [("bf16", 1.0, 1.0, 1.0),
         ("f16", 1.0, 1.0, 1.0),                             # inner products past the largest f16
         ("f16", 2.0 ** -17, 2.0 ** -17, 2.0 ** 10)]         # and such as f16 cannot hold, all of whose bits are below its smallest
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


def products_of_any_size(v, down, up, ids):
    """(up (down v_t), down v_t) of each row's adapter, in 64 bits: down [n][rank][C], up [n][C'][rank]"""
    low = torch.zeros(v.shape[0], down.shape[1], dtype=torch.float64, device="cuda")
    out = torch.zeros(v.shape[0], up.shape[1], dtype=torch.float64, device="cuda")
    for a in range(N):
        low[ids == a] = v[ids == a] @ down[a].t()
        out[ids == a] = low[ids == a] @ up[a].t()
    return out, low


def products(v, down, up, ids):
    out, low = products_of_any_size(v, down, up, ids)
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


@pytest.mark.parametrize("T", [4096, 20512])
def test_first_steps_of_an_adapter_in_f16(T):
    """B just after its start at zero, small gradients: every element of dA is rounded once, to 2^-11 of it or 2^-25, and its sum in fp32 has an error of 2^-21 of the
    magnitudes' sum."""
    ci, co, r = 256, 512, 16
    desc, dtype, w, _, one = setting(T, ci, co, "f16")
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (s * torch.randn(T, c, generator=g, device="cuda", dtype=torch.float64) for s, c in ((1.0, ci), (1e-4, co)))
    A, Bm = (s * torch.randn(N, *c, generator=g, device="cuda", dtype=torch.float64) for s, c in ((ci ** -0.5, (r, ci)), (1e-3, (co, r))))
    x, dy, A, Bm = (t.to(dtype) for t in (x, dy, A, Bm))
    ids = torch.zeros(T, dtype=torch.int32, device="cuda")
    y, low = B.snn_adapters_forward(desc, x, w, ids, A, Bm, one)
    dx, dA, dB = B.snn_adapters_backward(desc, x, low, dy, w, ids, A, Bm, one)
    dlow, S = dy.double() @ Bm[0].double(), dy.double().abs() @ Bm[0].double().abs()
    want = dlow.t() @ x.double()
    assert 1e-7 < float(dlow.abs().mean()) < 1e-5
    bound = 2.0 ** -11 * want.norm() + 2.0 ** -25 * want.numel() ** 0.5 + 2.0 ** -21 * (S.t() @ x.double().abs()).norm()
    assert float((dA[0].double() - want).norm()) <= float(bound)
    assert not bool(dA[1:].any()) and not bool(dB[1:].any())


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("rank", [16, 64])
def test_rows_of_very_different_sizes(rank, name):
    """Gradients of outputs that grow and shrink by 2^36 from chunk to chunk of an adapter's rows: what the largest contribute is as precise as if they were alone."""
    T, ci, co = 2000, 136, 264
    desc, dtype, w, _, one = setting(T, ci, co, name)
    g = torch.Generator(device="cuda").manual_seed(2)
    size = torch.exp2(torch.tensor([-18, -6, 2, 9, -15, 0, 12, -18], dtype=torch.float64, device="cuda")).repeat_interleave(250)[:, None]
    x, dy = (torch.randn(T, c, generator=g, device="cuda", dtype=torch.float64) for c in (ci, co))
    A, Bm = (torch.randn(N, *c, generator=g, device="cuda", dtype=torch.float64) for c in ((rank, ci), (co, rank)))
    x, dy, A, Bm = (t.to(dtype) for t in (x, dy * size, A / 2 ** 8, Bm / 2 ** 8))
    for order in (torch.arange(T, device="cuda"), torch.arange(T - 1, -1, -1, device="cuda")):
        xo, dyo = x[order].contiguous(), dy[order].contiguous()
        ids = torch.ones(T, dtype=torch.int32, device="cuda")
        y, low = B.snn_adapters_forward(desc, xo, w, ids, A, Bm, one)
        _, dA, dB = B.snn_adapters_backward(desc, xo, low, dyo, w, ids, A, Bm, one)
        u, tiny = (2.0 ** -8, 0.0) if name == "bf16" else (2.0 ** -11, 2.0 ** -25)
        dlow, S = dyo.double() @ Bm[1].double(), dyo.double().abs() @ Bm[1].double().abs()
        want = dlow.t() @ xo.double()
        assert bool(((dA[1].double() - want).abs() <= u * want.abs() + 2.0 ** -21 * (S.t() @ xo.double().abs()) + tiny).all())
        lo, S = xo.double() @ A[1].double().t(), xo.double().abs() @ A[1].double().abs().t()
        want = dyo.double().t() @ lo
        assert bool(((dB[1].double() - want).abs() <= u * want.abs() + 2.0 ** -21 * (dyo.double().abs().t() @ S) + tiny).all())


@pytest.mark.parametrize("name", sorted(TYPES))
@pytest.mark.parametrize("rank", [8, 72])
@pytest.mark.parametrize("T, ci, co", SHAPES)
def test_an_infinite_inner_product_gives_infinities(T, ci, co, rank, name):
    print("case", T, ci, co, rank, name, flush=True)
    desc, dtype, w, _, one = setting(T, ci, co, name)
    ids = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    ids[T // 2], ids[T // 2 + 1:] = 1, 0                     # (one row of the adapter with an infinite weight)
    x, A, Bm = numbers(1, (T, ci), ci) / 128, near_pairs(2, (N, rank, ci)) / 128, turned(opposites(3, (N, rank, co)))
    dy = torch.ones(T, co, dtype=torch.float64, device="cuda") * torch.tensor([1.0, -1.0], device="cuda").repeat(co // 2)
    A[1, 5, 7] = float("inf")
    want, low = products_of_any_size(x, A, Bm, ids)
    y, got = B.snn_adapters_forward(desc, x.to(dtype), w, ids, A.to(dtype), Bm.to(dtype), one)
    row = T // 2
    assert bool(got[row, 5].isposinf()) and bool(want[row].isinf().all())
    assert torch.equal(y[row].double(), want[row]) and bool(y[torch.arange(T, device="cuda") != row].isfinite().all())
    Bm[1, :, 3] *= float("inf")
    A[1, 5, 7] = 1.0
    _, low = products_of_any_size(x, A, Bm, ids)
    low[row, 5] = float("inf")
    dy = dy * torch.sign(Bm[1, :, 3]) * torch.sign(dy)       # (so that the infinities of the inner product have one sign)
    dx, dA, dB = B.snn_adapters_backward(desc, x.to(dtype), low.float(), dy.to(dtype), w, ids, A.to(dtype), Bm.to(dtype), one)
    assert torch.equal(dx[row].isinf(), torch.ones(ci, dtype=torch.bool, device="cuda")) and bool((dx[row] > 0).all())
    assert bool((dA[1, 3] == float("inf")).all()) and bool(dA[1, [r for r in range(rank) if r != 3]].isfinite().all())
    assert torch.equal(dB[1, :, 5].double(), dy[row] * float("inf")) and bool(dB[1][:, [r for r in range(rank) if r != 5]].isfinite().all())
    # the other adapter's gradients are finite where their formula's values are (sums of many rows can be past f16's range)
    rows = ids == 0
    _, dlow = products_of_any_size(dy, turned(Bm), turned(A), ids)
    for got, want in ((dA, dlow[rows].t() @ x[rows]), (dB, dy[rows].t() @ low[rows])):
        assert torch.equal(got[0].isfinite(), want.to(dtype).isfinite()) and not bool(got[0].isnan().any())
