"""The native part of the binding and the general one make the same calls of a network's ends."""
import pytest
import torch

from paper_2110_09195_amd import binding as B

pytestmark = pytest.mark.gpu


def _calls(dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    rows, V, C, k = 37, 500, 72, 5
    desc = B.make_vocab_desc(V, C, B._LINEAR_DTYPE.index(dtype))
    table = torch.randn(V, C, generator=g, device="cuda").to(dtype)
    wide = torch.randn(rows, C + 8, generator=g, device="cuda").to(dtype)
    x, ids = wide[:, :C], torch.randint(-1, V, (rows,), generator=g, device="cuda").int()
    listed, logits = torch.randint(0, V, (rows, k), generator=g, device="cuda").int(), torch.randn(rows, k, generator=g, device="cuda")
    dloss, held = torch.rand(rows, generator=g, device="cuda"), torch.randn(V, C, generator=g, device="cuda").to(dtype)
    lse, lse2 = B.snn_cross_entropy_forward(desc, x, table, ids)[1], B.snn_distill_forward(desc, x, table, listed, logits, 2.0)[1]
    return [
        ("embedding_forward", lambda f: f(desc, table, ids, 0.5, None)), ("embedding_forward", lambda f: f(desc, table, ids, 2, torch.zeros_like(wide)[:, :C])),
        ("embedding_grad", lambda f: f(desc, x, ids, 0.5, None, False, None)), ("embedding_grad", lambda f: f(desc, x, ids, 0.5, held.clone(), True, None)),
        ("cross_entropy_forward", lambda f: f(desc, x, table, ids, None, None, None)),
        ("cross_entropy_forward", lambda f: f(desc, x, table, ids, torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"),
                                              torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))),
        ("cross_entropy_backward", lambda f: f(desc, x, table, ids, lse, dloss, None, None, False, None)),
        ("cross_entropy_backward", lambda f: f(desc, x, table, ids, lse, dloss, False, held.clone(), True, None)),
        ("cross_entropy_backward", lambda f: f(desc, x, table, ids, lse, dloss, torch.zeros_like(wide)[:, :C], False, False, None)),
        ("distill_forward", lambda f: f(desc, x, table, listed, logits, 2.0, None, None, None, None)),
        ("distill_backward", lambda f: f(desc, x, table, listed, logits, 2.0, lse2, dloss, None, None, False, None)),
        ("distill_backward", lambda f: f(desc, x, table, listed, logits, 2, lse2, dloss, None, held.clone(), True, None)),
    ]


def _tensors(r):
    return [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_native_and_general_calls_agree(dtype, monkeypatch):
    assert B._fast is not None
    for n, (name, call) in enumerate(_calls(dtype)):
        native = call(getattr(B._fast, name))
        assert native is not False, (n, name)                         # (the ordinary case is taken natively)
        with monkeypatch.context() as mp:
            mp.setattr(B, "_fast", None)
            general = call(getattr(B, "snn_" + name))
        a, b = _tensors(native), _tensors(general)
        assert len(a) == len(b) and all(torch.equal(s, t) for s, t in zip(a, b)), (n, name)


def test_what_is_not_ordinary_is_left_to_the_general_call():
    desc, table = B.make_vocab_desc(50, 40), torch.randn(50, 40, device="cuda").bfloat16()
    x, target = torch.randn(6, 40, device="cuda").bfloat16(), torch.zeros(6, dtype=torch.int32, device="cuda")
    for args in ((desc, x.half(), table, target), (desc, x, table[:49], target), (desc, x, table, target.long()), (desc, x, table, target[:5]),
                 (desc, x.t().contiguous().t(), table, target), (desc, x.cpu(), table, target), (B.make_linear_desc(1, 40, 50, 4), x, table, target)):
        assert B._fast.cross_entropy_forward(*args, None, None, None) is False
    for args in ((desc, x.half(), table, target), (desc, x, table[:49], target), (desc, x, table, target.long()), (desc, x, table, target[:5])):
        with pytest.raises((TypeError, ValueError)):
            B.snn_cross_entropy_forward(*args)
    with pytest.raises(ValueError):
        B.snn_embedding_grad(desc, x, target, accumulate=True)         # nothing to add to
    with pytest.raises((ValueError, B.SnnError)):
        B.snn_cross_entropy_backward(desc, x, table, target, torch.zeros(6, device="cuda"), torch.zeros(6, device="cuda"), dx=False, dtable=False)
    with pytest.raises(B.SnnError):
        B.snn_distill_forward(desc, x, table, target.view(6, 1), torch.zeros(6, 1, device="cuda"), 0.0)
    with pytest.raises(B.SnnError):
        B.snn_cross_entropy_forward(desc, x, table, target, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
