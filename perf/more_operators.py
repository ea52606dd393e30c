"""The two ends of a network over tokens, as programs use them, in cases that can be timed and compared.

A table [V][C] of 16-bit values turns tokens into rows of channels at one end, and rows into logits over the vocabulary, whose
loss is what training follows, at the other.  A case names a path and its sizes:

  embed       tokens' rows of the table, times a scale
  embed_grad  the table's gradient from those of the rows
  loss        softmax cross entropy of rows against their targets (scoring: the losses and the logarithms of the sums alone)
  loss_step   the same in training: and the gradients of rows and table
  distill     the divergence of the softmax at a temperature from a teacher's, of which a row has the top logits alone; and the
              rows' own logits of the same tokens
  distill_step  the same in training

Targets and tokens outside 0 .. V - 1 belong to nothing: rows of zeros, losses of zero, no gradient.

`run` has two forms: elementary torch operations in 32 bits, and (with `own`) the calls of
`paper_2110_09195_amd.binding`.  `exact` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one token of one request: the smallest call
        {"name": "embed-token", "path": "embed", "rows": 1, "V": 32768, "C": 4096, "none": 0.0, "dtype": "bf16"},
        # a training batch's tokens, some of them padding
        {"name": "embed-batch", "path": "embed", "rows": 16384, "V": 131072, "C": 4096, "none": 0.05, "dtype": "bf16"},
        # the table's gradient from a training batch; tokens as frequent as words are
        {"name": "embed-grad", "path": "embed_grad", "rows": 16384, "V": 131072, "C": 4096, "none": 0.05, "skew": 1.0, "dtype": "bf16"},
        # a small table of odd sizes, every row of which has many tokens
        {"name": "embed-grad-odd", "path": "embed_grad", "rows": 7001, "V": 401, "C": 1032, "none": 0.3, "skew": 1.2, "dtype": "f16"},
        # how likely one token was: the whole table is read for one row
        {"name": "loss-token", "path": "loss", "rows": 1, "V": 131072, "C": 4096, "none": 0.0, "dtype": "bf16"},
        # short answers scored, an odd vocabulary
        {"name": "loss-answers", "path": "loss", "rows": 75, "V": 50021, "C": 2056, "none": 0.0, "dtype": "f16"},
        # texts scored, their first halves given
        {"name": "loss-texts", "path": "loss", "rows": 4096, "V": 65536, "C": 2048, "none": 0.5, "dtype": "bf16"},
        # a training step of a large model's last layer on a full batch: the largest work
        {"name": "loss-step", "path": "loss_step", "rows": 8192, "V": 131072, "C": 4096, "none": 0.02, "dtype": "bf16"},
        # a training step on answers, most rows being questions; nothing a multiple of a tile
        {"name": "loss-step-odd", "path": "loss_step", "rows": 1501, "V": 30011, "C": 1032, "none": 0.6, "dtype": "f16"},
        # a student's step on what a teacher answered, of which 64 logits a row were kept
        {"name": "distill-step", "path": "distill_step", "rows": 4096, "V": 65536, "C": 2048, "k": 64, "temperature": 2.0, "none": 0.1,
         "dtype": "bf16"},
        # a short batch of odd sizes with few logits
        {"name": "distill-step-odd", "path": "distill_step", "rows": 333, "V": 10007, "C": 776, "k": 11, "temperature": 1.5,
         "none": 0.3, "dtype": "f16"},
        # how far a student is from its teacher on a few rows
        {"name": "distill-rows", "path": "distill", "rows": 16, "V": 32768, "C": 2048, "k": 20, "temperature": 1.0, "none": 0.0,
         "dtype": "bf16"},
    ]


def draw(rng):
    def log_int(lo, hi, step=1):
        v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
        return max(lo, min(hi, int(round(v / step)) * step))

    path = rng.choice(["embed", "embed_grad", "loss", "loss", "loss_step", "loss_step", "distill", "distill_step"])
    case = {"path": path, "none": rng.choice([0.0, 0.05, 0.3, 0.7]), "dtype": rng.choice(["bf16", "bf16", "f16"])}
    # vocabularies that are multiples of many powers of two, or any number; channels of wide layers, or any multiple of 8
    case["V"] = 1024 * log_int(2, 128) if rng.random() < 0.4 else log_int(300, 131072)
    case["C"] = 2 ** rng.randint(9, 12) if rng.random() < 0.4 else log_int(256, 2900, 8)
    if path in ("embed", "embed_grad"):
        case["rows"] = log_int(1, 16384) if path == "embed" else log_int(64, 16384)
        if path == "embed_grad":
            case["skew"] = round(rng.uniform(0.0, 1.3), 2)
        return case
    most = min(8192, 2 ** 29 // case["V"])
    case["rows"] = log_int(64, max(most, 128)) if path.endswith("_step") else log_int(1, most)
    if path.startswith("distill"):
        case["k"] = log_int(1, 128)
        case["temperature"] = rng.choice([1.0, 1.5, 2.0, 4.0])
    return case


# ---- inputs ------------------------------------------------------------------------------------------------------

def _none(case):
    """Whether a row belongs to nothing: the same rows for every seed, so that the work of a case is one number; never all of them."""
    rng = random.Random("%(rows)d %(V)d %(C)d %(none)s" % case)
    return [False] + [rng.random() < case["none"] for _ in range(case["rows"] - 1)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, T, V, C = DTYPES[case["dtype"]], case["rows"], case["V"], case["C"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    none = torch.tensor(_none(case), device="cuda")
    s = {"case": case}
    if case["path"] != "embed_grad":
        s["table"] = normal(V, C).mul_(C ** -0.5).to(dtype)
    if case["path"].startswith("embed"):
        if "skew" in case:              # the r-th most frequent token as often as a power of r says; which token that is, is random
            p = torch.arange(1, V + 1, device="cuda").double() ** -case["skew"]
            rank = torch.searchsorted(p.cumsum(0) / p.sum(), uniform(T).double()).clamp(max=V - 1)
            ids = torch.randperm(V, generator=gen, device="cuda")[rank]
        else:
            ids = torch.randint(0, V, (T,), generator=gen, device="cuda")
        s["ids"] = torch.where(none, -1, ids).to(torch.int32)
        s["scale"] = math.sqrt(C)
        if case["path"] == "embed_grad":
            s["dy"] = (0.01 * normal(T, C)).to(dtype)
    else:
        # rows after a norm, each leaning towards the token that will be its target or its teacher's first, from not at all to nearly surely
        first = torch.randint(0, V, (T,), generator=gen, device="cuda")
        lean = uniform(T, 1) * 1.5 * math.log(V)
        s["x"] = (normal(T, C) + lean * s["table"][first].float()).to(dtype)
        if case["path"].startswith("loss"):
            s["target"] = torch.where(none, -1, first).to(torch.int32)
        else:
            k = case["k"]
            others = (first[:, None] + 1 + torch.randint(0, V - k, (T, 1), generator=gen, device="cuda")
                      + torch.arange(k, device="cuda") * max(1, (V - 1) // (2 * k))) % V
            others[:, 0] = first
            s["ids"] = torch.where(none[:, None], -1, others).to(torch.int32)
            s["logits"] = (8 - 3 * torch.log1p(torch.arange(k, device="cuda").float()) + 0.5 * normal(T, k)).contiguous()
            s["temperature"] = case["temperature"]
        if case["path"].endswith("_step"):
            # (with f16 a loss is trained times a power of two, so that small gradients are numbers of the type)
            s["dloss"] = (0.5 + uniform(T)) * ((4096.0 if dtype == torch.float16 else 1.0) / T)
    if own:
        from paper_2110_09195_amd import binding as B
        s["lib"] = B
        s["desc"] = B.make_vocab_desc(V, C, {"bf16": B.SNN_DTYPE_BF16, "f16": B.SNN_DTYPE_F16}[case["dtype"]])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    path = s["case"]["path"]
    if own:
        B, d = s["lib"], s["desc"]
        if path == "embed":
            return B.snn_embedding_forward(d, s["table"], s["ids"], s["scale"])
        if path == "embed_grad":
            return B.snn_embedding_grad(d, s["dy"], s["ids"], s["scale"])
        if path.startswith("loss"):
            loss, lse = B.snn_cross_entropy_forward(d, s["x"], s["table"], s["target"])
            if path == "loss":
                return loss, lse
            return loss, lse, *B.snn_cross_entropy_backward(d, s["x"], s["table"], s["target"], lse, s["dloss"])
        teacher = s["ids"], s["logits"], s["temperature"]
        loss, lse, picked = B.snn_distill_forward(d, s["x"], s["table"], *teacher)
        if path == "distill":
            return loss, lse, picked
        return loss, lse, picked, *B.snn_distill_backward(d, s["x"], s["table"], *teacher, lse, s["dloss"])
    if path == "embed":
        return _plain_embed(s)
    if path == "embed_grad":
        return _plain_embed_grad(s)
    return _plain_loss(s) if path.startswith("loss") else _plain_distill(s)


def _plain_embed(s):
    ids = s["ids"].long()
    ok = (ids >= 0) & (ids < s["table"].shape[0])
    rows = s["table"][torch.where(ok, ids, 0)].float() * s["scale"]
    return torch.where(ok[:, None], rows, 0.0).to(s["table"].dtype)


def _plain_embed_grad(s):
    ids, V = s["ids"].long(), s["case"]["V"]
    ids = torch.where((ids >= 0) & (ids < V), ids, V)
    grad = torch.zeros(V + 1, s["dy"].shape[1], device="cuda")
    grad.index_add_(0, ids, s["dy"].float())
    return (grad[:V] * s["scale"]).to(s["dy"].dtype)


def _plain_softmax(s, ok, temperature):
    """(rows that count, table in fp32; logits over the temperature; the logarithm of their exponentials' sum, 0 in rows that do not count)"""
    x, w = torch.where(ok[:, None], s["x"], 0).float(), s["table"].float()
    z = x @ w.t()
    if temperature != 1.0:
        z /= temperature
    top = z.amax(1, keepdim=True)
    lse = ((z - top).exp().sum(1, keepdim=True)).log() + top
    return x, w, z, lse


def _plain_loss(s):
    target, V = s["target"].long(), s["table"].shape[0]
    ok = (target >= 0) & (target < V)
    target = torch.where(ok, target, 0)[:, None]
    x, w, z, lse = _plain_softmax(s, ok, 1.0)
    loss = torch.where(ok, (lse - z.gather(1, target))[:, 0], 0.0)
    out = loss, torch.where(ok, lse[:, 0], 0.0)
    if "dloss" not in s:
        return out
    g = torch.where(ok, s["dloss"], 0.0)[:, None]
    z = (z - lse).exp_() * g
    z.scatter_add_(1, target, -g)
    return *out, (z @ w).to(s["x"].dtype), (z.t() @ x).to(s["table"].dtype)


def _plain_distill(s):
    ids, V, tau = s["ids"].long(), s["table"].shape[0], s["temperature"]
    listed = (ids >= 0) & (ids < V)
    ok = listed.any(1)
    ids = torch.where(listed, ids, 0)
    t = torch.where(listed, s["logits"] / tau, float("-inf"))
    e = torch.where(listed, (t - torch.where(ok, t.amax(1), 0.0)[:, None]).exp(), 0.0)
    q = e / torch.where(ok, e.sum(1), 1.0)[:, None]
    x, w, z, lse = _plain_softmax(s, ok, tau)
    logq = torch.where(q > 0, q.log(), 0.0)
    picked = z.gather(1, ids)
    loss = torch.where(ok, (q * (logq - picked + lse)).sum(1), 0.0)
    out = loss, torch.where(ok, lse[:, 0], 0.0), torch.where(listed, picked * tau, 0.0)
    if "dloss" not in s:
        return out
    g = torch.where(ok, s["dloss"], 0.0)[:, None] / tau
    z = (z - lse).exp_() * g
    z.scatter_add_(1, ids, -g * q)
    return *out, (z @ w).to(s["x"].dtype), (z.t() @ x).to(s["table"].dtype)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------

def _exact_embed(s, case):
    ids, V = s["ids"].long(), case["V"]
    mine = ((ids >= 0) & (ids < V)).nonzero().flatten()
    if case["path"] == "embed":
        y = torch.zeros(case["rows"], case["C"], dtype=torch.float64, device="cuda")
        y[mine] = s["scale"] * s["table"].double()[ids[mine]]
        return y
    # the rows of a token lie next to each other once sorted: differences of running sums over 256 channels at a time
    order = mine[torch.argsort(ids[mine], stable=True)]
    count = torch.bincount(ids[order], minlength=V)
    end = count.cumsum(0)
    grad = torch.empty(V, case["C"], dtype=torch.float64, device="cuda")
    for c in range(0, case["C"], 256):
        run = torch.zeros(order.numel() + 1, min(256, case["C"] - c), dtype=torch.float64, device="cuda")
        run[1:] = s["dy"][order, c:c + 256].double().cumsum(0)
        grad[:, c:c + 256] = s["scale"] * (run[end] - run[end - count])
    return grad


def exact(case, seed):
    s = prepare(case, seed)
    if case["path"].startswith("embed"):
        return _exact_embed(s, case)
    V, T, C = case["V"], case["rows"], case["C"]
    tau = float(case.get("temperature", 1.0))
    if "target" in s:
        ids = s["target"].long()[:, None]
        weight = ((ids >= 0) & (ids < V)).double()
    else:
        ids = s["ids"].long()
        teacher = s["logits"].double() / tau
        teacher[(ids < 0) | (ids >= V)] = -math.inf
        weight = torch.softmax(teacher, 1).nan_to_num(0.0)          # (a row without any: not a number)
    rows = (weight.sum(1) > 0).nonzero().flatten()                  # those that count; the others stay zero
    x, ids, weight = s["x"].double()[rows], ids[rows].clamp(0, V - 1), weight[rows]
    step = max(1024, 2 ** 27 // max(1, T))                          # of the vocabulary
    lse = torch.full((rows.numel(),), -math.inf, dtype=torch.float64, device="cuda")
    for v in range(0, V, step):
        z = x @ s["table"][v:v + step].double().t() / tau
        lse = torch.logaddexp(lse, torch.logsumexp(z, 1))
    picked = torch.stack([(x * s["table"][ids[:, j]].double()).sum(1) for j in range(ids.shape[1])], 1) / tau
    loss, whole = torch.zeros(2, T, dtype=torch.float64, device="cuda").unbind(0)
    loss[rows] = lse - (weight * picked).sum(1) + torch.special.xlogy(weight, weight).sum(1)
    whole[rows] = lse
    out = loss, whole
    if "logits" in s:                                               # the student's own logits of the tokens that the teacher lists
        theirs = torch.zeros(T, case["k"], dtype=torch.float64, device="cuda")
        theirs[rows] = picked * tau
        out += (torch.where((s["ids"] >= 0) & (s["ids"] < V), theirs, 0.0),)
    if "dloss" not in s:
        return out
    g = s["dloss"].double()[rows] / tau
    dx = torch.zeros(T, C, dtype=torch.float64, device="cuda")
    dw = torch.zeros(V, C, dtype=torch.float64, device="cuda")
    for v in range(0, V, step):
        w = s["table"][v:v + step].double()
        dz = torch.exp(x @ w.t() / tau - lse[:, None])
        for j in range(ids.shape[1]):
            at = ((ids[:, j] >= v) & (ids[:, j] < v + w.shape[0])).nonzero().flatten()
            dz[at, ids[at, j] - v] -= weight[at, j]
        dz *= g[:, None]
        dx[rows] += dz @ w
        dw[v:v + w.shape[0]] = dz.t() @ x
    return *out, dx, dw


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(case):
    T, V, C = case["rows"], case["V"], case["C"]
    used = case["rows"] - sum(_none(case))                          # rows that count
    if case["path"] == "embed":
        return {"bytes": 4 * T + 2 * min(used, V) * C + 2 * T * C, "flops": T * C}
    if case["path"] == "embed_grad":
        return {"bytes": 4 * T + 2 * used * C + 2 * V * C, "flops": used * C}
    k = case.get("k", 1)
    listed = (4 if "k" not in case else 12 * k) * T                 # targets; or tokens, the teacher's logits and the student's
    if not case["path"].endswith("_step"):
        return {"bytes": 2 * used * C + 2 * V * C + listed + 8 * T, "flops": 2 * used * C * V}
    return {"bytes": 2 * used * C + 2 * V * C + listed + 12 * T + 2 * T * C + 2 * V * C, "flops": 6 * used * C * V}
