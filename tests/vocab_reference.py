"""The ends of a network over tokens in 64 bits, element by element from their definitions, and how far the calls may be from them."""
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}          # half a step of a rounding, relative
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}                # and absolute, where values are no normal numbers
F32 = 2.0 ** -24


def embedding(table, ids, scale):
    ok = (ids >= 0) & (ids < table.shape[0])
    y = table.double()[torch.where(ok, ids, 0).long()] * scale
    return torch.where(ok[:, None], y, torch.zeros_like(y))


def by_token(dy, ids, V):
    """Sums, sums of magnitudes and numbers of rows, by token."""
    ok = ((ids >= 0) & (ids < V)).nonzero().flatten()
    out = [torch.zeros(V, dy.shape[1], dtype=torch.float64, device=dy.device) for _ in range(2)]
    rows = dy.double()[ok]
    out[0].index_add_(0, ids[ok].long(), rows)
    out[1].index_add_(0, ids[ok].long(), rows.abs())
    return out[0], out[1], torch.bincount(ids[ok].long(), minlength=V).double()


class Loss:
    """Cross entropy (logits None, ids [rows]) or distillation (ids, logits [rows][k]) of x against a table; gradients for dloss.  Every quantity
    comes with a bound of the error that a call may have:

      z        products of 16-bit values are exact in 32 bits; C sums, each off by half a step of at most the magnitudes' sum
      exp, log 2^-21 relative each (the arguments' rounding among it), sums of positive terms a step for each of the terms that follow each other
      dz       the type's half step of its own magnitude, and p's error
      dx, dw   dz's errors times the other factor, a 32-bit sum over the contracted axis, one rounding
    """

    def __init__(self, x, table, ids, logits=None, temperature=1.0, dloss=None):
        T, C = x.shape
        V = table.shape[0]
        dev, unit, tiny = x.device, UNIT[x.dtype], TINY[x.dtype]
        ids = ids.long().view(T, -1)
        listed = (ids >= 0) & (ids < V)
        if logits is None:
            q = listed.double()
        else:
            t = torch.where(listed, logits.double() / temperature, torch.full((), float("-inf"), dtype=torch.float64, device=dev))
            q = torch.softmax(t, 1)
            q = torch.where((t > float("-inf")).any(1, keepdim=True) | t.isnan().any(1, keepdim=True), q, torch.zeros_like(q))
        self.counts = (q.sum(1) != 0)
        rows = self.counts.nonzero().flatten()
        xd, wd, ids, q, listed = x.double()[rows], table.double(), torch.where(listed, ids, 0)[rows], q[rows], listed[rows]
        z = xd @ wd.t()
        ez = (C * F32) * (xd.abs() @ wd.abs().t())                     # of the logits
        lse = torch.logsumexp(z / temperature, 1)
        steps = (512 + V / 128) * F32
        top = z.abs().amax(1) / temperature
        elog = ez.amax(1) / temperature + steps + 2.0 ** -21 * (1 + top)
        picked = z.gather(1, ids)
        terms = torch.special.xlogy(q, q) + q * (lse[:, None] - picked / temperature)

        def whole(v):
            out = torch.zeros((T,) + v.shape[1:], dtype=torch.float64, device=dev)
            out[rows] = v
            return out
        self.loss, self.lse = whole(terms.sum(1)), whole(lse)
        # (shares: exp of what is rounded in 32 bits)
        share = 0 if logits is None else 2.0 ** -20 * (1 + (logits.double().abs().nan_to_num(0, 0, 0).amax(1)[rows] / temperature))
        magnitude = (q * (q.clamp(min=1e-300).log().abs() + lse.abs()[:, None] + picked.abs() / temperature)).sum(1)
        self.loss_error = whole(2 * elog + (share + 2.0 ** -20) * magnitude)
        self.lse_error = whole(elog + F32 * lse.abs())
        self.picked = whole(torch.where(listed, picked, torch.zeros_like(picked)))
        self.picked_error = whole(ez.gather(1, ids))
        if dloss is None:
            return
        g = dloss.double()[rows] / temperature
        p = torch.exp(z / temperature - lse[:, None])
        dz = p.clone()
        dz.scatter_add_(1, ids, -q)
        dz *= g[:, None]
        ep = p * (ez / temperature + elog[:, None] + 2.0 ** -20 * (2 + top[:, None]))
        if logits is not None:
            ep.scatter_add_(1, ids, q * share[:, None])
        else:
            ep.scatter_add_(1, ids, q * 2.0 ** -22)
        g = g.abs()[:, None]
        edz = unit * dz.abs() + g * ep * (1 + unit)
        if x.dtype == torch.float16:
            edz = edz + 2.0 ** -39 * g.max() if g.numel() else edz
        del ep, ez, p, z
        self.dx = whole(dz @ wd)
        self.dx_error = whole(edz @ wd.abs() + (V + 64) * F32 * (dz.abs() @ wd.abs())) + unit * self.dx.abs() + tiny
        self.dx_error *= 1 + unit
        self.dw = dz.t() @ xd
        self.dw_error = (edz.t() @ xd.abs() + (T + 64) * F32 * (dz.abs().t() @ xd.abs()) + unit * self.dw.abs() + tiny) * (1 + unit)


def within(got, want, error, name):
    off = (got.double() - want).abs()
    bad = ~(off <= error)                                              # (what is not a number is never within)
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError("%s: %d of %d off, at %s by %g of at most %g (value %g)" % (
            name, int(bad.sum()), bad.numel(), at, float(off[tuple(at)]), float(error[tuple(at)]), float(want[tuple(at)])))
