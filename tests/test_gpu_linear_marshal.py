"""The native part of the binding of the projections' calls: it gives what the general part gives, and what that part refuses is refused with the
same error."""
import pytest
import torch

from paper_2110_09195_amd import binding as B

pytestmark = pytest.mark.gpu


def _calls():
    """(name, arguments, position -> arguments that are refused there)"""
    T, ci, co, n, r = 20, 72, 40, 3, 8
    d = B.make_linear_desc(2, ci, co, 16, B.SNN_DTYPE_F16)
    one = B.make_linear_desc(1, ci, co, 16, B.SNN_DTYPE_F16)
    g = torch.Generator(device="cuda").manual_seed(3)
    cb, idx = torch.arange(32, device="cuda").to(torch.int16).view(2, 16), torch.randint(0, 16, (2, co, ci // 8), device="cuda", generator=g).to(torch.int16)
    alpha = torch.rand(2, co, device="cuda", generator=g).half()
    w = B.snn_linear_prepare(d, cb, idx, alpha)
    w1 = B.snn_linear_prepare(one, cb[:1].contiguous(), idx[:1].contiguous(), alpha[:1].contiguous())
    x, dy = torch.randn(T, ci, device="cuda", generator=g).half(), torch.randn(T, co, device="cuda", generator=g).half()
    off = torch.tensor([0, 7, T], dtype=torch.int32, device="cuda")
    bad_x = [x.float(), x.cpu(), x[:, :64], torch.randn(ci, T, device="cuda").half().t(), x[0], 3, None]
    yield "snn_linear_forward", [d, x, w, off], {0: [None, one], 1: bad_x, 2: [w[:256], w.cpu(), None], 3: [None, off.long(), off[:2].contiguous(), off.cpu()]}
    yield "snn_linear_input_grad", [d, dy, w, off], {1: [dy.float(), dy[:, :32]], 2: [w[:256]], 3: [None, off.long()]}
    yield "snn_checkpoint_store", [x], {0: [x.float(), x.cpu(), x[:, :60], x[0], None]}
    kept = B.snn_checkpoint_store(x)
    yield "snn_checkpoint_restore", [kept, torch.float16], {0: [(kept[0], kept[1][:, :3].contiguous()), (kept[0].cpu(), kept[1]), (kept[0].short(), kept[1])],
                                                            1: [torch.float32, None]}
    A, Bm, scale = torch.randn(n, r, ci, device="cuda", generator=g).half(), torch.randn(n, co, r, device="cuda", generator=g).half(), torch.rand(n, device="cuda")
    ids = torch.randint(-1, n, (T,), device="cuda", generator=g).int()
    yield "snn_adapters_forward", [one, x, w1, ids, A, Bm, scale], {0: [d, None], 1: bad_x, 2: [w1[:256]], 3: [ids.long(), ids[:5].contiguous(), None],
                                                                    4: [A.float(), A[:, :5].contiguous(), A[0]], 5: [Bm.float(), Bm[:2].contiguous()],
                                                                    6: [scale.half(), scale[:2].contiguous()]}


def _flat(r):
    return list(r) if isinstance(r, tuple) else [r]


def _general(monkeypatch, name, args, **kw):
    with monkeypatch.context() as mp:
        mp.setattr(B, "_fast", None)
        return getattr(B, name)(*args, **kw)


def test_native_and_general_calls_agree(monkeypatch):
    B.lib()
    assert B._fast is not None
    for name, args, bad in _calls():
        print(name, flush=True)
        assert getattr(B._fast, name[4:])(*(list(args[0]) + [1, None] if name.endswith("restore") else args + [None] * {"snn_checkpoint_store": 2, "snn_adapters_forward": 3}.get(name, 1))) is not False
        want = _flat(_general(monkeypatch, name, args))
        got = _flat(getattr(B, name)(*args))
        assert len(got) == len(want) and all(a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b) for a, b in zip(got, want))
        for at, values in bad.items():
            for v in values:
                wrong = list(args)
                wrong[at] = v
                with pytest.raises(Exception) as general:
                    _general(monkeypatch, name, wrong)
                with pytest.raises(general.type) as native:
                    getattr(B, name)(*wrong)
                assert str(native.value) == str(general.value), (name, at)


def test_given_outputs_and_rows_apart():
    name, (d, x, w, off), _ = next(_calls())
    want = B.snn_linear_forward(d, x, w, off)
    wide = torch.zeros(20, 88, device="cuda").half()
    wide[:, :72] = x
    out = torch.zeros(20, 56, device="cuda").half()
    got = B.snn_linear_forward(d, wide[:, :72], w, off, y=out[:, 8:48])
    assert got.data_ptr() == out[:, 8:48].data_ptr() and torch.equal(out[:, 8:48], want) and not bool(out[:, :8].any()) and not bool(out[:, 48:].any())
    p = torch.nn.Parameter(x)
    y = B.snn_linear_forward(d, p, w, off)
    assert torch.equal(y, want) and not y.requires_grad
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = B.snn_linear_forward(d, x, w, off)
    side.synchronize()
    assert torch.equal(y, want)


def test_given_outputs_are_taken_natively_or_refused():
    calls = {name: args for name, args, _ in _calls()}
    x = calls["snn_checkpoint_store"][0]
    q, e = B.snn_checkpoint_store(x)
    q1, e1 = torch.empty_like(q), torch.empty_like(e)
    assert B._fast.checkpoint_store(x, q1, e1) is not False and torch.equal(q, q1) and torch.equal(e, e1)
    wide = torch.zeros(20, 88, device="cuda").half()
    assert B._fast.checkpoint_restore(q, e, B.SNN_DTYPE_F16, wide[:, 8:80]) is not False
    assert torch.equal(wide[:, 8:80], B.snn_checkpoint_restore((q, e), torch.float16)) and not bool(wide[:, :8].any()) and not bool(wide[:, 80:].any())
    args = calls["snn_adapters_forward"]
    y, low = B.snn_adapters_forward(*args)
    y1, low1, ws = torch.zeros_like(y), torch.zeros_like(low), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    assert B._fast.adapters_forward(*args, y1, low1, ws) is not False and torch.equal(y, y1) and torch.equal(low, low1)
    for name, a, kw in (("snn_checkpoint_store", [x], {"q": q1[:3].contiguous()}), ("snn_checkpoint_store", [x], {"e": e1.short()}),
                        ("snn_checkpoint_restore", [(q, e), torch.float16], {"x": wide[:7, :72]}), ("snn_adapters_forward", args, {"low": low1.double()}),
                        ("snn_adapters_forward", args, {"workspace": ws[:16]}), ("snn_adapters_forward", args, {"workspace": ws.cpu()})):
        with pytest.raises(Exception):
            getattr(B, name)(*a, **kw)
