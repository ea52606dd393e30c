"""What the calls on projections of real-valued activations refuse (CPU only: every call is refused before any device work)."""
import ctypes

import pytest
import torch

from paper_2110_09195_amd import binding as B

BAD, UNSUP, WS = B.SNN_ERR_INVALID_ARG, B.SNN_ERR_UNSUPPORTED, B.SNN_ERR_WORKSPACE
P = 1 << 20            # an address that no refused call looks at
BIG = 1 << 40


def desc(**kw):
    d = B.make_linear_desc(2, 64, 32, 16, B.SNN_DTYPE_BF16)
    for k, v in kw.items():
        setattr(d, k, v)
    return ctypes.byref(d)


def adapters(**kw):
    a = B.snn_adapters(4, 16, P, P, P)
    for k, v in kw.items():
        setattr(a, k, v)
    return ctypes.byref(a)


def call(name, args, **change):
    """The entry point with its arguments by name, some of them changed."""
    a = dict(args, **change)
    return getattr(B.lib(), name)(*a.values())


ROWS = dict(desc=desc(), x=P, ldx=64, rows=8, offsets=P, weights=P, wb=BIG, y=P, ldy=32, stream=None)
GRAD = dict(desc=desc(), x=P, ldx=64, dy=P, lddy=32, rows=8, offsets=P, weights=P, wb=BIG, dw=P, dalpha=P, ws=P, wsb=BIG, stream=None)
GRAD8 = dict(desc=desc(), q=P, e=P, dy=P, lddy=32, rows=8, offsets=P, weights=P, wb=BIG, dw=P, dalpha=P, ws=P, wsb=BIG, stream=None)
FWD = dict(desc=desc(groups=1), ad=adapters(), x=P, ldx=64, rows=8, adapter=P, weights=P, wb=BIG, y=P, ldy=32, low=P, ws=P, wsb=BIG, stream=None)
BWD = dict(desc=desc(groups=1), ad=adapters(), x=P, ldx=64, low=P, dy=P, lddy=32, rows=8, adapter=P, weights=P, wb=BIG, dx=P, lddx=64, dA=P,
           dB=P, ws=P, wsb=BIG, stream=None)
BWD8 = dict(desc=desc(groups=1), ad=adapters(), q=P, e=P, low=P, dy=P, lddy=32, rows=8, adapter=P, weights=P, wb=BIG, dx=P, lddx=64, dA=P,
            dB=P, ws=P, wsb=BIG, stream=None)
PREP = dict(desc=desc(), codebook=P, idx=P, alpha=P, weights=P, wb=BIG, stream=None)
STORE = dict(x=P, ldx=64, rows=8, C=64, dtype=0, q=P, e=P, stream=None)
RESTORE = dict(q=P, e=P, rows=8, C=64, dtype=0, x=P, ldx=64, stream=None)
CALLS = {"snn_linear_forward": ROWS, "snn_linear_weight_grad": GRAD, "snn_linear_weight_grad_checkpoint": GRAD8, "snn_adapters_forward": FWD,
         "snn_adapters_backward": BWD, "snn_adapters_backward_checkpoint": BWD8, "snn_linear_prepare": PREP, "snn_checkpoint_store": STORE,
         "snn_checkpoint_restore": RESTORE,
         "snn_linear_input_grad": dict(desc=desc(), dy=P, lddy=32, rows=8, offsets=P, weights=P, wb=BIG, dx=P, lddx=64, stream=None)}

BAD_DESC = [dict(groups=0), dict(groups=1025), dict(C_in=0), dict(C_in=60), dict(C_in=65544), dict(C_out=4), dict(C_out=65544), dict(C_out=36),
            dict(K=0), dict(K=257), dict(dtype=2), dict(dtype=-1)]


@pytest.mark.parametrize("name", [n for n in CALLS if "checkpoint_" not in n or n.endswith("_checkpoint")])
def test_descriptors(name):
    assert call(name, CALLS[name], desc=None) == BAD
    for bad in BAD_DESC:
        assert call(name, CALLS[name], desc=desc(**bad)) == BAD, bad
    assert B.lib().snn_linear_weights_bytes(desc(C_in=60)) == 0 and B.lib().snn_linear_weights_bytes(None) == 0
    assert B.lib().snn_linear_weight_grad_workspace_bytes(desc(K=0), 8, 0) == 0 and B.lib().snn_linear_weight_grad_workspace_bytes(desc(), -1, 1) == 0
    assert B.lib().snn_adapters_workspace_bytes(desc(groups=1), adapters(), 8, 3) == 0 and B.lib().snn_adapters_workspace_bytes(desc(groups=1), adapters(), 8, 2) > 0
    assert B.lib().snn_adapters_workspace_bytes(desc(), adapters(), 8, 1) == 0            # two groups


@pytest.mark.parametrize("name", sorted(CALLS))
def test_pointers_distances_and_counts(name):
    args = CALLS[name]
    for key in args:
        if key in ("x", "y", "dy", "dx", "low", "adapter", "offsets", "dw", "dA", "dB", "q", "e", "codebook", "idx", "alpha", "ad"):
            if key == "low" and name == "snn_adapters_forward":
                continue                                     # (not wanted)
            assert call(name, args, **{key: None}) == BAD, key
        if key in ("x", "y", "dy", "dx", "dw", "dA", "dB", "q", "low"):
            assert call(name, args, **{key: P + 8}) == BAD, key
        if key.startswith("ld"):
            for v in (args[key] - 8, args[key] + 4, (1 << 20) + 8, -64, 0):
                assert call(name, args, **{key: v}) == BAD, (key, v)
        if key == "rows":
            assert call(name, args, rows=-1) == BAD and call(name, args, rows=1 << 28) == BAD


@pytest.mark.parametrize("name", sorted(CALLS))
def test_weights_and_workspaces(name):
    args = CALLS[name]
    for ptr, size in (("weights", "wb"), ("ws", "wsb")):
        if ptr in args:
            for change in ({ptr: None}, {ptr: P + 128}, {size: 64}, {size: 0}):
                assert call(name, args, **change) == WS, change


def test_adapters():
    for name, args in (("snn_adapters_forward", FWD), ("snn_adapters_backward", BWD), ("snn_adapters_backward_checkpoint", BWD8)):
        for bad in (dict(n=0), dict(n=65537), dict(rank=0), dict(rank=12), dict(rank=136), dict(A=None), dict(B=None), dict(scale=None), dict(A=P + 2)):
            assert call(name, args, ad=adapters(**bad)) == BAD, bad
        assert call(name, args, desc=desc()) == UNSUP


def test_checkpoints():
    for name, args in (("snn_checkpoint_store", STORE), ("snn_checkpoint_restore", RESTORE)):
        for bad in (dict(C=0), dict(C=60), dict(C=65544), dict(dtype=2)):
            assert call(name, args, **bad) == BAD, bad


def test_binding_checks_its_tensors():
    d = B.make_linear_desc(1, 64, 32, 16, B.SNN_DTYPE_BF16)
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for f in (lambda: B.snn_linear_forward(d, x, None), lambda: B.snn_linear_input_grad(d, x, None), lambda: B.snn_checkpoint_store(x),
              lambda: B.snn_linear_prepare(d, x, x, x), lambda: B.snn_linear_weight_grad(d, x, x, None),
              lambda: B.snn_adapters_forward(d, x, None, None, None, None, None)):
        with pytest.raises(TypeError):
            f()
    with pytest.raises(ValueError):
        B.snn_linear_forward(B.make_linear_desc(1, 64, 32, 16, 5), x, None)
