"""Layers over tokens from the library's projections: experts that are trained in sub-bit form, and a fixed projection with an adapter a request.

    python -m paper_2110_09195_amd.token_layers

trains both for some steps towards random teachers of their own kind, and serves the adapted projection token by token.
"""
import torch
from torch.autograd.function import once_differentiable

from . import binding as B

_CODES = {torch.bfloat16: B.SNN_DTYPE_BF16, torch.float16: B.SNN_DTYPE_F16}


class _Experts(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, alpha, codebook8, offsets, keep_8_bits):
        groups, c_out, c_in = w.shape
        desc = B.make_linear_desc(groups, c_in, c_out, codebook8.shape[1], _CODES[x.dtype])
        idx = torch.stack([B.snn_project_vectors8(w[g], codebook8[g]) for g in range(groups)]).view(groups, c_out, c_in // 8)
        weights = B.snn_linear_prepare(desc, codebook8, idx, alpha.to(x.dtype))
        kept = B.snn_checkpoint_store(x) if keep_8_bits else (x,)
        ctx.save_for_backward(weights, offsets, *kept)
        ctx.desc = desc
        return B.snn_linear_forward(desc, x, weights, offsets, y=torch.zeros(x.shape[0], c_out, dtype=x.dtype, device=x.device))

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        weights, offsets, *kept = ctx.saved_tensors
        dy = dy.contiguous()
        dx = B.snn_linear_input_grad(ctx.desc, dy, weights, offsets, dx=torch.zeros(dy.shape[0], ctx.desc.C_in, dtype=dy.dtype, device=dy.device))
        # (straight through: the gradient of the +-1 weights is that of the real ones)
        dw, dalpha = B.snn_linear_weight_grad(ctx.desc, kept[0] if len(kept) == 1 else tuple(kept), dy, weights, offsets)
        return dx, dw, dalpha, None, None, None


def experts(x, w, alpha, codebook8, offsets, keep_8_bits=True):
    """x [rows][C_in] in 16 bits, rows sorted by expert as offsets (int32 [experts + 1]) says (rows before the first and behind the last expert's: outputs and
    gradients of zero), through projections whose weights are the nearest
    members of the experts' subsets codebook8 (int16 [experts][K]) to the vectors of 8 of w (float32 [experts][C_out][C_in]), times
    alpha (float32 [experts][C_out]).  Differentiable (once) in x, w (straight through) and alpha; x is kept in 8 bits or as it is."""
    return _Experts.apply(x, w, alpha, codebook8, offsets, keep_8_bits)


class _Adapted(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, A, Bm, scale, adapter, desc, weights, keep_8_bits):
        A, Bm = A.to(x.dtype), Bm.to(x.dtype)
        y, low = B.snn_adapters_forward(desc, x, weights, adapter, A, Bm, scale)
        ctx.save_for_backward(A, Bm, scale, adapter, weights, low, *(B.snn_checkpoint_store(x) if keep_8_bits else (x,)))
        ctx.desc = desc
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        A, Bm, scale, adapter, weights, low, *kept = ctx.saved_tensors
        dx, dA, dB = B.snn_adapters_backward(ctx.desc, kept[0] if len(kept) == 1 else tuple(kept), low, dy.contiguous(), weights, adapter, A, Bm, scale)
        return dx, dA.float(), dB.float(), None, None, None, None, None


def adapted(x, A, Bm, scale, adapter, desc, weights, keep_8_bits=True):
    """x [rows][C_in] in 16 bits through the projection that snn_linear_prepare laid out as weights and, beside it, each row's adapter
    (int32 [rows], outside 0 .. n - 1: none): A float32 [n][rank][C_in], Bm float32 [n][C_out][rank], scale float32 [n].
    Differentiable (once) in x, A and Bm; scale is a constant."""
    if scale.requires_grad:
        raise ValueError("scale has no gradient here: detach it, or put what is learnt into A or Bm")
    return _Adapted.apply(x, A, Bm, scale, adapter, desc, weights, keep_8_bits)


def by_expert(expert, n):
    """expert [rows] of 0 .. n - 1 -> (order of the rows by expert, offsets int32 [n + 1])."""
    order = torch.argsort(expert, stable=True)
    offsets = torch.zeros(n + 1, dtype=torch.int32, device=expert.device)
    offsets[1:] = torch.bincount(expert, minlength=n).cumsum(0)
    return order, offsets


def _random_codebook(groups, K, g):
    return torch.stack([torch.randperm(256, generator=g, device="cuda")[:K] for _ in range(groups)]).to(torch.int16)


def train_experts(steps=60, rows=1500, n=5, c_in=512, c_out=256, K=32, dtype=torch.bfloat16, seed=0):
    """Losses of the steps, towards experts whose weights are members of the same subsets."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codebook8 = _random_codebook(n, K, g)
    desc = B.make_linear_desc(n, c_in, c_out, K, _CODES[dtype])
    idx = torch.randint(0, K, (n, c_out, c_in // 8), generator=g, device="cuda").to(torch.int16)
    teacher = B.snn_linear_prepare(desc, codebook8, idx, torch.full((n, c_out), c_in ** -0.5, device="cuda").to(dtype))
    w = (0.1 * torch.randn(n, c_out, c_in, generator=g, device="cuda")).requires_grad_()
    alpha = torch.full((n, c_out), 0.5 * c_in ** -0.5, device="cuda", requires_grad=True)
    optimizer, losses = torch.optim.Adam([{"params": [w], "lr": 1e-2}, {"params": [alpha], "lr": 1e-3}]), []
    for _ in range(steps):
        x = torch.randn(rows, c_in, generator=g, device="cuda").to(dtype)
        order, offsets = by_expert(torch.randint(0, n, (rows,), generator=g, device="cuda"), n)
        x = x[order]
        y = experts(x, w, alpha, codebook8, offsets)
        loss = (y.float() - B.snn_linear_forward(desc, x, teacher, offsets).float()).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    return [float(v) for v in losses]


def train_adapters(steps=60, rows=800, n=6, rank=16, c_in=512, c_out=256, K=32, dtype=torch.bfloat16, seed=0):
    """(losses of the steps, what serving needs), towards the same projection with other adapters."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    desc = B.make_linear_desc(1, c_in, c_out, K, _CODES[dtype])
    idx = torch.randint(0, K, (1, c_out, c_in // 8), generator=g, device="cuda").to(torch.int16)
    weights = B.snn_linear_prepare(desc, _random_codebook(1, K, g), idx, torch.full((1, c_out), c_in ** -0.5, device="cuda").to(dtype))

    def pair(b):
        return torch.randn(n, rank, c_in, generator=g, device="cuda") * c_in ** -0.5, torch.randn(n, c_out, rank, generator=g, device="cuda") * b
    scale = torch.full((n,), 2.0, device="cuda")
    want_A, want_B = (t.to(dtype) for t in pair(rank ** -0.5))
    A, Bm = (t.requires_grad_() for t in pair(0.0))
    optimizer, losses = torch.optim.Adam([A, Bm], lr=1e-2), []
    for _ in range(steps):
        x = torch.randn(rows, c_in, generator=g, device="cuda").to(dtype)
        adapter = torch.randint(-1, n, (rows,), generator=g, device="cuda").sort()[0].int()
        want, _ = B.snn_adapters_forward(desc, x, weights, adapter, want_A, want_B, scale)
        loss = (adapted(x, A, Bm, scale, adapter, desc, weights).float() - want.float()).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    return [float(v) for v in losses], (desc, weights, A.detach().to(dtype), Bm.detach().to(dtype), scale)


def serve(served, x, adapter):
    """One token of each request at a time: x [tokens][requests][C_in], adapter int32 [requests] -> y [tokens][requests][C_out].  Outputs and
    workspace are made once, as a server's loop keeps them."""
    desc, weights, A, Bm, scale = served
    tokens, requests, _ = x.shape
    y = torch.empty(tokens, requests, desc.C_out, dtype=x.dtype, device=x.device)
    low = torch.empty(requests, A.shape[1], device=x.device)
    size = B.snn_adapters_workspace_bytes(desc, B.snn_adapters(A.shape[0], A.shape[1], A.data_ptr(), Bm.data_ptr(), scale.data_ptr()), requests)
    workspace = torch.empty(size, dtype=torch.uint8, device=x.device)
    for t in range(tokens):
        B.snn_adapters_forward(desc, x[t], weights, adapter, A, Bm, scale, y=y[t], low=low, workspace=workspace)
    return y


def main():
    for name, losses in (("experts", train_experts()), ("adapters", train_adapters()[0])):
        print("%-8s loss %.4f -> %.4f in %d steps" % (name, losses[0], losses[-1], len(losses)))
    _, served = train_adapters(steps=5)
    x = torch.randn(64, 24, served[0].C_in, device="cuda").to(served[2].dtype)
    adapter = torch.arange(24, dtype=torch.int32, device="cuda") % 7
    y = serve(served, x, adapter)
    whole, _ = B.snn_adapters_forward(served[0], x.flatten(0, 1), served[1], adapter.repeat(64), *served[2:])
    print("served   64 tokens of 24 requests, at most %.4f from the same rows in one call" % (y.flatten(0, 1).float() - whole.float()).abs().max())


if __name__ == "__main__":
    main()
