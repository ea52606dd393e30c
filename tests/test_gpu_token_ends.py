"""The layers at the ends of a network over tokens: their gradients against automatic differentiation in 64 bits, and a network of all layers together."""
import pytest
import torch

from paper_2110_09195_amd import binding as B
from paper_2110_09195_amd import token_layers as TL
from vocab_reference import UNIT

pytestmark = pytest.mark.gpu


def _near(got, want, bound, name):
    err = (got.double() - want).norm() / want.norm()
    assert float(err) <= bound, (name, float(err))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("k", [0, 6])
def test_gradients(dtype, k):
    g = torch.Generator(device="cuda").manual_seed(3)
    rows, V, C, tau = 70, 300, 72, 2.0 if k else 1.0
    table = (torch.randn(V, C, generator=g, device="cuda") * 0.2).to(dtype).requires_grad_()
    ids = torch.randint(-1, V, (rows,), generator=g, device="cuda").int()
    x = torch.randn(rows, C, generator=g, device="cuda").to(dtype)
    weight = torch.rand(rows, generator=g, device="cuda")
    h = TL.embedded(ids, table, 3.0) + x
    some = ids >= 0
    td = table.detach().double().requires_grad_()
    e = torch.where(some[:, None], 3.0 * td[ids.clamp(min=0).long()], torch.zeros((), dtype=torch.float64, device="cuda"))
    hd = e + x.double() + (h.detach().double() - (e + x.double())).detach()          # (the rounded rows, differentiated as if they were not)
    z = hd @ td.t() / tau
    if k:
        listed, logits = torch.randint(0, V, (rows, k), generator=g, device="cuda").int(), torch.randn(rows, k, generator=g, device="cuda")
        loss = TL.distilled(h, table, listed, logits, tau)
        q = torch.softmax(logits.double() / tau, 1)
        want = (q * (q.log() - torch.log_softmax(z, 1).gather(1, listed.long()))).sum(1)
    else:
        target = torch.randint(0, V, (rows,), generator=g, device="cuda")
        loss = TL.cross_entropy(h, table, target.int())
        want = torch.nn.functional.cross_entropy(z, target, reduction="none")
    _near(loss.detach(), want.detach(), 1e-5, "loss")
    (loss * weight).sum().backward()
    (want * weight.double()).sum().backward()
    # Two gradients of the table, added.  The loss's: dz and the sum rounded.  The embedding's: from rows' gradients that carry dz's rounding and one of their
    # own, its sum rounded.  Autograd's sum of both rounded.  Each at most a unit of a norm that is at most the sum of theirs.
    parts = torch.autograd.grad((TL.cross_entropy(h.detach(), table, target.int()) if not k else TL.distilled(h.detach(), table, listed, logits, tau)).mul(weight).sum(), table)[0]
    size = (parts.double().norm() + (td.grad - parts.double()).norm()) / td.grad.norm()
    _near(table.grad, td.grad, 4 * UNIT[dtype] * float(size) + 1e-4, "dtable")


def test_only_what_is_needed():
    table = torch.randn(50, 40, device="cuda").bfloat16()
    x, target = torch.randn(9, 40, device="cuda").bfloat16().requires_grad_(), torch.arange(9, dtype=torch.int32, device="cuda")
    TL.cross_entropy(x, table, target).sum().backward()
    dx = x.grad.clone()
    t = table.clone().requires_grad_()
    TL.cross_entropy(x.detach(), t, target).sum().backward()
    x.grad = None
    both = table.clone().requires_grad_()
    TL.cross_entropy(x, both, target).sum().backward()
    assert torch.equal(x.grad, dx) and torch.equal(both.grad, t.grad)


def test_what_is_refused():
    table, x = torch.randn(50, 40, device="cuda").bfloat16(), torch.randn(9, 40, device="cuda").bfloat16()
    ids = torch.zeros(9, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        TL.distilled(x, table, ids, torch.zeros(9, 3, device="cuda", requires_grad=True))
    x.requires_grad_()
    target = ids[:, 0].contiguous()
    dx, = torch.autograd.grad(TL.cross_entropy(x, table, target).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        dx.sum().backward()


@pytest.mark.parametrize("k", [0, 5])
def test_a_captured_step(k):
    """Forward and backward captured together, no graph of an eager step over the same leaves living then, and replayed on changing inputs."""
    g = torch.Generator(device="cuda").manual_seed(5)
    rows, V, C = 200, 700, 136
    table = torch.randn(V, C, generator=g, device="cuda").bfloat16().requires_grad_()
    ids = torch.randint(-1, V, (rows,), generator=g, device="cuda").int()
    target = torch.randint(-1, V, (rows, k) if k else (rows,), generator=g, device="cuda").int()
    logits = torch.randn(rows, max(k, 1), generator=g, device="cuda")

    def step():
        h = TL.embedded(ids, table, 0.1)
        loss = TL.distilled(h, table, target, logits, 2.0) if k else TL.cross_entropy(h, table, target)
        return loss.detach(), *torch.autograd.grad(loss.mean(), table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for n in range(3):
        ids.copy_(torch.randint(-1, V, (rows,), generator=g, device="cuda"))
        target.copy_(torch.randint(-1, V, target.shape, generator=g, device="cuda"))
        graph.replay()
        got = [t.clone() for t in kept]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step())), n


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("k", [0, 9])
def test_a_network_trains(dtype, k):
    losses = TL.train_tokens(steps=4, rows=300, k=k, V=500, C=128, dtype=dtype)
    assert len(losses) == 4 and all(v == v and v >= 0 for v in losses)


def test_a_network_steps_as_its_layers_in_64_bits():
    """One step of tokens through table, experts, table again and loss: the gradient of the table that both ends share."""
    V, C, rows = 400, 128, 200
    (table, w, alpha), network = TL.token_network(V, C, n=3)
    ids = torch.randint(0, V, (rows,), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    order, h, t16 = network(ids)
    target = ids[order].flip(0)
    TL.cross_entropy(h, t16, target.int()).mean().backward()
    # the same network as the library's layers round it, the experts by their outputs' derivative
    t = t16.detach().double().requires_grad_()
    x = t[ids[order]] * C ** 0.5
    expert, eye = ids[order] % 3, torch.eye(C, device="cuda").to(t16.dtype)
    g = torch.Generator(device="cuda").manual_seed(0)
    cb = TL._random_codebook(3, 32, g)
    d = B.make_linear_desc(3, C, C, 32)
    idx = torch.stack([B.snn_project_vectors8(w[e].detach(), cb[e]) for e in range(3)]).view(3, C, C // 8)
    weights = B.snn_linear_prepare(d, cb, idx, alpha.detach().to(t16.dtype))
    each = torch.arange(4, dtype=torch.int32, device="cuda") * C
    W = B.snn_linear_forward(d, eye.repeat(3, 1), weights, each).double().view(3, C, C)
    out = torch.stack([x[i] + x[i] @ W[int(expert[i])] for i in range(rows)])
    out = out + (h.detach().double() - out).detach()
    loss = torch.nn.functional.cross_entropy(out @ t.t(), target)
    loss.backward()
    # (dz, the gradients of rows before and behind the experts, of their inputs, both of the table and their sum: seven roundings of parts that may cancel by
    # a factor of two)
    _near(table.grad, t.grad, 14 * UNIT[t16.dtype], "table")


def test_the_command_runs(capsys):
    TL.main()
    out = capsys.readouterr().out
    assert "tokens" in out and "taught" in out
