"""Projections of real-valued activations by sub-bit weights, as programs use them, in cases that can be timed and compared.

A projection's C_out x C_in weights are cut into vectors of 8 consecutive input channels, each a member of a subset of
{+-1}^8 and stored as its index; every output channel has a scale.  A case names a path and its sizes:

  forward        rows of several requests, sorted by expert, through the experts' projections
  step           a training step of the experts: weights laid out from new indices, outputs, and the gradients of inputs,
                 of the +-1 weights and of the scales; the inputs kept for the backward pass as they are or in 8 bits
  adapters       rows of many requests through one shared projection, each with its request's low-rank adapter beside it
  adapters_step  a training step of adapters beside a fixed projection: inputs kept in 8 bits, outputs, and the gradients
                 of inputs and adapters
  store          activations into their 8-bit form and back

`run` has two forms: elementary torch operations in 32 bits, and (with `own`) the calls of
`paper_2110_09195_amd.binding`.  `exact` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CHUNK = 32              # channels of a row that share an exponent in the 8-bit form


def listed():
    return [
        # one token of sixteen requests, each sent to two of many experts: latency, most experts idle
        {"name": "experts-token", "path": "forward", "rows": 32, "groups": 32, "C_in": 2048, "C_out": 1024, "K": 32,
         "skew": 0.5, "dtype": "bf16"},
        # prompts through wide experts, the popular ones with several times the rows of the others
        {"name": "experts-prompt", "path": "forward", "rows": 8192, "groups": 8, "C_in": 4096, "C_out": 4096, "K": 64,
         "skew": 0.7, "dtype": "bf16"},
        # many small experts, a few dozen rows each, nothing a multiple of a tile
        {"name": "experts-ragged", "path": "forward", "rows": 1537, "groups": 60, "C_in": 1032, "C_out": 1416, "K": 256,
         "skew": 1.0, "dtype": "f16"},
        # a training step of wide experts on a full batch: the largest work
        {"name": "experts-step", "path": "step", "rows": 16384, "groups": 8, "C_in": 4096, "C_out": 4096, "K": 32,
         "skew": 0.5, "checkpoint": False, "dtype": "bf16"},
        # a training step of small experts of odd sizes, inputs kept in 8 bits
        {"name": "experts-step-odd", "path": "step", "rows": 2999, "groups": 5, "C_in": 776, "C_out": 1304, "K": 16,
         "skew": 1.0, "checkpoint": True, "dtype": "f16"},
        # one token of one request: the smallest call
        {"name": "adapters-one", "path": "adapters", "rows": 1, "adapters": 8, "rank": 8, "C_in": 2048, "C_out": 2048,
         "K": 32, "bare": 0.0, "run": 1, "dtype": "f16"},
        # one token each of many requests, nearly all of them with an adapter of their own
        {"name": "adapters-token", "path": "adapters", "rows": 48, "adapters": 64, "rank": 16, "C_in": 4096, "C_out": 4096,
         "K": 64, "bare": 0.1, "run": 1, "dtype": "bf16"},
        # prompts of some hundred tokens each, a quarter of them without an adapter
        {"name": "adapters-prompt", "path": "adapters", "rows": 4096, "adapters": 12, "rank": 32, "C_in": 4096,
         "C_out": 4096, "K": 64, "bare": 0.25, "run": 150, "dtype": "bf16"},
        # several adapters trained at once on one batch
        {"name": "adapters-step", "path": "adapters_step", "rows": 8192, "adapters": 4, "rank": 64, "C_in": 4096,
         "C_out": 4096, "K": 32, "bare": 0.0, "run": 2048, "dtype": "bf16"},
        # the same at odd sizes, some rows without an adapter
        {"name": "adapters-step-odd", "path": "adapters_step", "rows": 1111, "adapters": 7, "rank": 24, "C_in": 1352,
         "C_out": 2056, "K": 128, "bare": 0.1, "run": 170, "dtype": "f16"},
        # the inputs of a wide layer on a full batch, kept for the backward pass
        {"name": "store-batch", "path": "store", "rows": 16384, "C_in": 8192, "dtype": "bf16"},
        # one short sequence, a last chunk of channels that is not whole
        {"name": "store-odd", "path": "store", "rows": 333, "C_in": 1000, "dtype": "f16"},
    ]


def draw(rng):
    def log_int(lo, hi, step=1):
        v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
        return max(lo, min(hi, int(round(v / step)) * step))

    def channels():             # powers of two as wide layers have them, or any multiple of 8
        return 2 ** rng.randint(9, 12) if rng.random() < 0.3 else log_int(512, 2900, 8)

    path = rng.choice(["forward", "forward", "step", "adapters", "adapters", "adapters_step", "store"])
    case = {"path": path, "dtype": rng.choice(["bf16", "bf16", "f16"])}
    if path == "store":
        case.update(rows=log_int(64, 16384), C_in=rng.choice([4096, 8192]) if rng.random() < 0.3 else log_int(256, 2900, 8))
        return case
    case.update(C_in=channels(), C_out=channels(), K=2 ** rng.randint(3, 8))
    if path in ("forward", "step"):
        case.update(rows=log_int(4, 8192) if path == "forward" else log_int(512, 16384), groups=log_int(2, 64),
                    skew=round(rng.uniform(0.0, 1.2), 2))
        if path == "step":
            case["groups"] = min(case["groups"], 12)
            case["checkpoint"] = rng.random() < 0.5
        return case
    case.update(rank=8 * rng.randint(1, 8), bare=rng.choice([0.0, 0.1, 0.3]))
    if path == "adapters":
        case["adapters"] = log_int(2, 64)
        if rng.random() < 0.5:
            case.update(rows=log_int(1, 64), run=1)
        else:
            case.update(rows=log_int(256, 4096), run=log_int(32, 512))
    else:
        case.update(rows=log_int(512, 8192), adapters=rng.randint(1, 8))
        case["run"] = case["rows"] // case["adapters"] + 1
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------

def group_rows(case):
    """Rows of each expert: drawn with popularities that fall as a power of the rank, so that some may have none."""
    rng = random.Random("%(rows)d %(groups)d %(skew)s" % case)
    weights = [1.0 / (r + 1) ** case["skew"] for r in range(case["groups"])]
    rng.shuffle(weights)
    counts = [0] * case["groups"]
    for g in rng.choices(range(case["groups"]), weights, k=case["rows"]):
        counts[g] += 1
    return counts


def row_adapters(case):
    """The adapter of each row (-1: none): requests of about `run` rows each, of random adapters.  A training step has its
    rows in the adapters' order."""
    rng = random.Random("%(rows)d %(adapters)d %(run)d %(bare)s" % case)
    ids = []
    while len(ids) < case["rows"]:
        n = 1 if case["run"] == 1 else max(1, int(case["run"] * rng.uniform(0.5, 1.5)))
        a = -1 if rng.random() < case["bare"] else rng.randrange(case["adapters"])
        ids += [a] * n
    ids = ids[:case["rows"]]
    return sorted(ids) if case["path"] == "adapters_step" else ids


def _inputs(case, seed):
    """The tensors that both forms and the definition start from."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    dtype, T, ci = DTYPES[case["dtype"]], case["rows"], case["C_in"]
    # channels of different sizes, a few much larger than the others, as after a norm
    channel = torch.exp(0.5 * normal(ci)) * (1.0 + 15.0 * (torch.rand(ci, generator=gen, device="cuda") < 0.01))
    s = {"x": (normal(T, ci) * channel).to(dtype)}
    if case["path"] == "store":
        return s
    co, G, K = case["C_out"], case.get("groups", 1), case["K"]
    s["codebook"] = torch.stack([torch.randperm(256, generator=gen, device="cuda")[:K] for _ in range(G)]).to(torch.int16)
    s["idx"] = torch.randint(0, K, (G, co, ci // 8), generator=gen, device="cuda").to(torch.int16)
    s["alpha"] = ((0.5 + torch.rand(G, co, generator=gen, device="cuda")) / math.sqrt(ci)).to(dtype)
    if case["path"] in ("step", "adapters_step"):
        s["dy"] = (0.1 * normal(T, co)).to(dtype)
    if "groups" in case:
        s["counts"] = group_rows(case)
        ends = [0]
        for n in s["counts"]:
            ends.append(ends[-1] + n)
        s["offsets"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    else:
        n, r = case["adapters"], case["rank"]
        ids = row_adapters(case)
        s["ids"] = ids
        s["adapter"] = torch.tensor(ids, dtype=torch.int32, device="cuda")
        s["A"] = (normal(n, r, ci) / math.sqrt(ci)).to(dtype)
        s["B"] = (0.1 * normal(n, co, r)).to(dtype)
        s["scale"] = 0.5 + 1.5 * torch.rand(n, generator=gen, device="cuda")
    return s


def _member_signs(codebook):
    """int16 [G][K] codes -> float [G][K][8]: element j of a member is bit 7 - j, set for +1."""
    shifts = torch.arange(7, -1, -1, device=codebook.device)
    return (((codebook.long().unsqueeze(-1) >> shifts) & 1) * 2 - 1).float()


def _signs(codebook, idx):
    """-> float [G][C_out][C_in] of +-1"""
    members = _member_signs(codebook)
    return torch.stack([members[g][idx[g].long()].flatten(1) for g in range(idx.shape[0])])


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2110_09195_amd import binding as B
        s["lib"] = B
        dt = {"bf16": B.SNN_DTYPE_BF16, "f16": B.SNN_DTYPE_F16}[case["dtype"]]
        if case["path"] != "store":
            s["desc"] = B.make_linear_desc(case.get("groups", 1), case["C_in"], case["C_out"], case["K"], dt)
            if case["path"] != "step":                      # (a step of the experts lays its new weights out itself)
                s["weights"] = B.snn_linear_prepare(s["desc"], s["codebook"], s["idx"], s["alpha"])
    elif case["path"] in ("forward", "adapters", "adapters_step"):
        s["W"] = _signs(s["codebook"], s["idx"])
    if "ids" in s:
        s["members"] = [(a, torch.tensor([t for t, b in enumerate(s["ids"]) if b == a], device="cuda"))
                        for a in sorted(set(s["ids"])) if a >= 0]
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    return (_RUN_OWN if own else _RUN_PLAIN)[case["path"]](s)


def _own_forward(s):
    return s["lib"].snn_linear_forward(s["desc"], s["x"], s["weights"], offsets=s["offsets"])


def _own_step(s):
    B, d = s["lib"], s["desc"]
    weights = B.snn_linear_prepare(d, s["codebook"], s["idx"], s["alpha"])
    kept = B.snn_checkpoint_store(s["x"]) if s["case"]["checkpoint"] else s["x"]
    y = B.snn_linear_forward(d, s["x"], weights, offsets=s["offsets"])
    dx = B.snn_linear_input_grad(d, s["dy"], weights, offsets=s["offsets"])
    dw, dalpha = B.snn_linear_weight_grad(d, kept, s["dy"], weights, offsets=s["offsets"])
    return y, dx, dw, dalpha


def _own_adapters(s):
    y, _ = s["lib"].snn_adapters_forward(s["desc"], s["x"], s["weights"], s["adapter"], s["A"], s["B"], s["scale"])
    return y


def _own_adapters_step(s):
    B, d = s["lib"], s["desc"]
    kept = B.snn_checkpoint_store(s["x"])
    y, low = B.snn_adapters_forward(d, s["x"], s["weights"], s["adapter"], s["A"], s["B"], s["scale"])
    dx, dA, dB = B.snn_adapters_backward(d, kept, low, s["dy"], s["weights"], s["adapter"], s["A"], s["B"], s["scale"])
    return y, dx, dA, dB


def _own_store(s):
    B = s["lib"]
    return B.snn_checkpoint_restore(B.snn_checkpoint_store(s["x"]), s["x"].dtype)


def _split(t, counts):
    return torch.split(t, counts)


def _plain_rows(x, W, alpha, counts, dtype):
    y = [xg.float() @ W[g].t() * alpha[g].float() for g, xg in enumerate(_split(x, counts))]
    return torch.cat(y).to(dtype)


def _plain_forward(s):
    return _plain_rows(s["x"], s["W"], s["alpha"], s["counts"], s["x"].dtype)


def _plain_kept(x):
    """The values that the 8-bit form stands for: chunks of channels share the power of two that makes the largest finite
    magnitude one of 64 .. 128, elements are rounded to whole numbers of at most 127; what is not finite becomes NaN."""
    T, C = x.shape
    n = (C + CHUNK - 1) // CHUNK
    v = torch.nn.functional.pad(x.float(), (0, n * CHUNK - C)).view(T, n, CHUNK)
    finite = torch.isfinite(v)
    top = torch.where(finite, v.abs(), torch.zeros_like(v)).amax(-1, keepdim=True)
    exponent = torch.frexp(top)[1] - 7                       # (frexp: magnitudes of 0.5 .. 1)
    exponent = torch.where(top == 0, torch.full_like(exponent, -126), exponent.clamp(min=-126))
    unit = ((exponent + 127) << 23).to(torch.int32).view(torch.float32)
    q = (v / unit).round().clamp(-127, 127)
    kept = torch.where(finite, q * unit, torch.full_like(q, float("nan")))
    return kept.view(T, -1)[:, :C]


def _plain_step(s):
    dtype = s["x"].dtype
    W = _signs(s["codebook"], s["idx"])
    y = _plain_rows(s["x"], W, s["alpha"], s["counts"], dtype)
    kept = _plain_kept(s["x"]) if s["case"]["checkpoint"] else s["x"]
    dx, dw, dalpha = [], [], []
    for g, (xg, dyg) in enumerate(zip(_split(kept, s["counts"]), _split(s["dy"], s["counts"]))):
        dyg, a = dyg.float(), s["alpha"][g].float()
        dx.append((dyg * a) @ W[g])
        grad = dyg.t() @ xg.float()
        dw.append(grad * a[:, None])
        dalpha.append((grad * W[g]).sum(1))
    return y, torch.cat(dx).to(dtype), torch.stack(dw), torch.stack(dalpha)


def _plain_adapters_f32(s, lows=None):
    x, W, alpha = s["x"].float(), s["W"][0], s["alpha"][0].float()
    y = x @ W.t() * alpha
    if len(s["ids"]) <= 64:                                  # single tokens: every row with its own adapter
        has = s["adapter"] >= 0
        a = s["adapter"].clamp(min=0).long()
        low = (s["A"][a].float() * x[:, None, :]).sum(-1) * s["scale"][a][:, None]
        return y + torch.where(has[:, None], (s["B"][a].float() * low[:, None, :]).sum(-1), torch.zeros_like(y))
    for a, rows in s["members"]:
        low = x[rows] @ s["A"][a].float().t()
        if lows is not None:
            lows[a] = low
        y[rows] += s["scale"][a] * (low @ s["B"][a].float().t())
    return y


def _plain_adapters(s):
    return _plain_adapters_f32(s).to(s["x"].dtype)


def _plain_adapters_step(s):
    dtype, lows = s["x"].dtype, {}
    y = _plain_adapters_f32(s, lows).to(dtype)
    kept, dy = _plain_kept(s["x"]), s["dy"].float()
    dx = (dy * s["alpha"][0].float()) @ s["W"][0]
    dA, dB = torch.zeros_like(s["A"], dtype=torch.float32), torch.zeros_like(s["B"], dtype=torch.float32)
    for a, rows in s["members"]:
        g = dy[rows] * s["scale"][a]
        dlow = g @ s["B"][a].float()
        dx[rows] += dlow @ s["A"][a].float()
        dA[a] = dlow.t() @ kept[rows]
        dB[a] = g.t() @ lows[a]
    return y, dx.to(dtype), dA.to(dtype), dB.to(dtype)


def _plain_store(s):
    return _plain_kept(s["x"]).to(s["x"].dtype)


_RUN_PLAIN = {"forward": _plain_forward, "step": _plain_step, "adapters": _plain_adapters,
              "adapters_step": _plain_adapters_step, "store": _plain_store}
_RUN_OWN = {"forward": _own_forward, "step": _own_step, "adapters": _own_adapters, "adapters_step": _own_adapters_step,
            "store": _own_store}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def _exact_weights(codes, idx):
    """One matrix of +-1 in 64 bits, element by element: w[o][8 v + j] = 2 bit(7 - j) - 1 of the code that idx[o][v] names."""
    code = codes[idx.long()].long()
    w = torch.empty(idx.shape[0], idx.shape[1] * 8, dtype=torch.float64, device=idx.device)
    for j in range(8):
        w[:, j::8] = torch.where((code & (1 << (7 - j))) != 0, 1.0, -1.0).double()
    return w


def _exact_kept(x):
    x = x.double()
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], CHUNK):
        part = x[:, c:c + CHUNK]
        ok = torch.isfinite(part)
        top = torch.where(ok, part, torch.zeros_like(part)).abs().max(1, keepdim=True).values
        unit = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -120))) - 6)
        # (log2 of a value just below a power of two may round up to it)
        unit = torch.where(top < 64 * unit, unit / 2, unit).clamp(min=2.0 ** -126)
        out[:, c:c + CHUNK] = torch.where(ok, (part / unit).round().clamp(-127, 127) * unit, torch.full_like(part, float("nan")))
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if case["path"] == "store":
        return _exact_kept(s["x"])
    x, T = s["x"].double(), case["rows"]
    train = "dy" in s
    y = torch.zeros(T, case["C_out"], dtype=torch.float64, device="cuda")
    if train:
        dy, dx = s["dy"].double(), torch.zeros_like(x)
        kept = _exact_kept(s["x"]) if case.get("checkpoint", True) else x
    dws, dalphas, start = [], [], 0
    for g, n in enumerate(s.get("counts", [T])):
        w, alpha = _exact_weights(s["codebook"][g], s["idx"][g]), s["alpha"][g].double()
        rows = slice(start, start + n)
        start += n
        y[rows] = (x[rows] @ w.t()) * alpha
        if train:
            dx[rows] = dy[rows] @ (alpha[:, None] * w)
        if case["path"] == "step":
            grad = dy[rows].t() @ kept[rows]
            dws.append(alpha[:, None] * grad)
            dalphas.append((w * grad).sum(1))
    if case["path"] == "step":
        return y, dx, torch.stack(dws), torch.stack(dalphas)
    if case["path"] == "forward":
        return y
    dA, dB = torch.zeros_like(s["A"], dtype=torch.float64), torch.zeros_like(s["B"], dtype=torch.float64)
    for a in range(case["adapters"]):
        rows = (s["adapter"] == a).nonzero().flatten()
        if rows.numel() == 0:
            continue
        A, Bm, c = s["A"][a].double(), s["B"][a].double(), s["scale"][a].double()
        y[rows] += c * (x[rows] @ A.t()) @ Bm.t()
        if train:
            dx[rows] += c * (dy[rows] @ Bm) @ A
            dA[a] = c * (dy[rows] @ Bm).t() @ kept[rows]
            dB[a] = c * dy[rows].t() @ (x[rows] @ A.t())
    return (y, dx, dA, dB) if train else y


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(case):
    T, ci = case["rows"], case["C_in"]
    stored = T * (ci + (ci + CHUNK - 1) // CHUNK)            # a byte an element and one for each chunk
    if case["path"] == "store":
        return {"bytes": 2 * (2 * T * ci + stored), "flops": 4 * T * ci}
    co = case["C_out"]
    product = 2 * T * ci * co
    io = 2 * T * (ci + co)
    if case["path"] == "forward":
        used = sum(1 for n in group_rows(case) if n)
        return {"bytes": io + used * (ci * co // 8 + 2 * co), "flops": product}
    if case["path"] == "step":
        G = case["groups"]
        kept = stored if case["checkpoint"] else 0
        return {"bytes": 2 * io + kept + G * (2 * case["K"] + ci * co // 4 + 2 * co) + G * co * (4 * ci + 4),
                "flops": 3 * product}
    ids = row_adapters(case)
    r, n = case["rank"], len(set(a for a in ids if a >= 0))
    with_adapter = sum(1 for a in ids if a >= 0)
    shared = ci * co // 8 + 2 * co + 4 * T + 4 * n
    low = 2 * with_adapter * r * (ci + co)
    if case["path"] == "adapters":
        return {"bytes": io + shared + 2 * n * r * (ci + co), "flops": product + low}
    return {"bytes": 2 * io + stored + 2 * shared + 2 * (n + case["adapters"]) * r * (ci + co),
            "flops": 2 * product + 3 * low}
