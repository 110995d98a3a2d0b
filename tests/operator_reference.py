"""The router operators and the 8-bit products in 64 bits, straight from their definitions, and the bounds on what 32-bit
arithmetic may add (test infrastructure)."""
import torch

U = 2.0 ** -24          # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounding(dtype, ref):
    """What rounding ref to dtype may change: half a step, and half a step of the subnormal numbers (or what fp32 loses there)."""
    return half_step(dtype) * ref.abs() + torch.finfo(dtype).smallest_normal * half_step(dtype) + 1e-37


def probabilities(x, act):
    """x: float64 [T, E]; NaN counts as -inf.  Softmax (logits of +inf share the row) or shares of the sigmoids."""
    x = torch.where(torch.isnan(x), -torch.inf, x)
    if act == "softmax":
        top = x == torch.inf
        x = torch.where(top.any(1, keepdim=True), torch.where(top, 0.0, -torch.inf).to(x), x)
        p = torch.softmax(x, 1)
    else:
        p = torch.softmax(torch.nn.functional.logsigmoid(x), 1)
    return torch.nan_to_num(p, nan=0.0)


def topk(x, k, act, renorm, live=None):
    """Row by row, on the host -> idx, weights (float64)."""
    x = x.double().cpu()
    x = torch.where(torch.isnan(x), -torch.inf, x)
    T, E = x.shape
    live = T if live is None else live
    idx = torch.full((T, k), -1, dtype=torch.int64)
    for t in range(min(T, live)):
        by = sorted(range(E), key=lambda e: (-x[t, e].item(), e))
        picks = [e for e in by if x[t, e] > -torch.inf][:k]
        idx[t, :len(picks)] = torch.tensor(picks, dtype=torch.int64)
    return idx, weights_of(x, idx, act, renorm)


def weights_of(x, idx, act, renorm):
    """Weights of chosen experts as a function of the logits (float64, differentiable where all is finite)."""
    there = idx >= 0
    at = idx.clamp(min=0)
    if renorm:
        chosen = torch.zeros(x.shape, dtype=torch.bool, device=x.device)
        chosen[torch.arange(x.shape[0], device=x.device)[:, None].expand_as(idx)[there], idx[there]] = True
        p = probabilities(torch.where(chosen, x, -torch.inf), act)
    else:
        p = probabilities(x, "softmax") if act == "softmax" else torch.sigmoid(x)
    return torch.where(there, p.gather(1, at), 0.0)


def topk_grad(x, idx, act, renorm, d_weights):
    """d_logits, and the sum of the sizes of the terms that each entry is made of."""
    x = torch.where(torch.isnan(x), -torch.inf, x.double())
    there = idx >= 0
    w = weights_of(x, idx, act, renorm)
    g = torch.where(there, d_weights.double(), 0.0)
    s, size = (g * w).sum(1, keepdim=True), (g * w).abs().sum(1, keepdim=True)
    d, big = torch.zeros_like(x), torch.zeros_like(x)
    if act == "softmax" and not renorm:
        p = probabilities(x, "softmax") * there.any(1, keepdim=True)
        at = idx.clamp(min=0)
        gx, ga = torch.zeros_like(x).scatter_add_(1, at, g), torch.zeros_like(x).scatter_add_(1, at, g.abs())
        return torch.where(p > 0, p * (gx - s), 0.0), p * (ga + size)
    part = w * (g - s) if renorm else w * g
    psize = w * (g.abs() + size)
    if act == "sigmoid":
        rest = torch.where(there, torch.sigmoid(-x.gather(1, idx.clamp(min=0))), 0.0)
        part, psize = part * rest, psize * rest
    at = idx.clamp(min=0)
    return d.scatter_add_(1, at, torch.where(there, part, 0.0)), big.scatter_add_(1, at, torch.where(there, psize, 0.0))


def order(idx, E):
    """Stable counting sort on the host -> offsets, order, position."""
    flat = idx.reshape(-1).tolist()
    lists = [[i for i, e in enumerate(flat) if e == want] for want in range(E)]
    offsets = [0]
    for one in lists:
        offsets.append(offsets[-1] + len(one))
    out = [i for one in lists for i in one]
    position = [-1] * len(flat)
    for at, i in enumerate(out):
        position[i] = at
    return offsets, out + [-1] * (len(flat) - len(out)), position


def balance(x, idx, seg, act):
    """float64 logits, idx, segment offsets (a list) -> loss, counts, mean_p, rows."""
    T, E = x.shape
    p = probabilities(x, act)
    loss, counts, mean, rows = [], [], [], []
    for a, b in zip(seg[:-1], seg[1:]):
        part = idx[a:b]
        named = (part >= 0) & (part < E)
        on = named.any(1)
        c = torch.bincount(part[named].long(), minlength=E)[:E]
        m = (p[a:b] * on[:, None]).sum(0) / max(int(on.sum()), 1)
        loss.append(E * (c.double() / max(int(c.sum()), 1) * m).sum())
        counts.append(c)
        mean.append(m)
        rows.append(int(on.sum()))
    return torch.stack(loss), torch.stack(counts), torch.stack(mean), rows


def balance_grad(x, idx, seg, act, d_loss):
    """d_logits and the sizes of its terms."""
    T, E = x.shape
    x = torch.where(torch.isnan(x), -torch.inf, x)
    p = probabilities(x, act)
    d, size = torch.zeros_like(x), torch.zeros_like(x)
    for s, (a, b) in enumerate(zip(seg[:-1], seg[1:])):
        part = idx[a:b]
        named = (part >= 0) & (part < E)
        on = named.any(1)
        n = int(on.sum())
        if n == 0:
            continue
        c = torch.bincount(part[named].long(), minlength=E)[:E].double()
        f = (c / c.sum())[None]
        pi = p[a:b] * on[:, None]
        k = d_loss[s].double() * E / n
        inner = (f * pi).sum(1, keepdim=True)
        slope = pi if act == "softmax" else pi * torch.sigmoid(-x[a:b])
        d[a:b] = torch.where(pi > 0, k * slope * (f - inner), 0.0)
        size[a:b] = torch.where(pi > 0, k.abs() * slope * (f + inner), 0.0)
    return d, size


def reach(x):
    """How far finite logits of a row lie apart, and from 0: an exponent's argument is off by half a step of that."""
    x = x.double()
    x = x[torch.isfinite(x)]
    return 0.0 if x.numel() == 0 else float((x.max() - x.min()).abs().clamp(min=x.abs().max()))


def rel_p(x, act):
    """Relative bound on a probability.  e^d, d = x - top, is a power of 2 whose argument is off by half a step of d and by what log2 e
    is off, or, of sizes beyond 10^38, by half a step of d twice; two steps of the power itself: (2 |d| + 4) U at most.  The sum of up
    to 512 such terms is off by their mean, weighted by p -- sum p |d| is at most the entropy, ln 512 < 6.3 -- that is 17 U, and by 24 U
    of additions (a tree behind 16 serial ones); reciprocal and products 4 U.  A sigmoid's own steps (an addition and a reciprocal,
    3 U) stand in the place of the difference's."""
    return (2 * (reach(x) + 8) + 32) * U


def codes_of(x):
    """8-bit codes of the rows of x (float64, exact quotients) and their largest sizes."""
    x = x.double()
    a = x.abs().amax(1)
    return torch.where(a[:, None] > 0, torch.round(127 * x / torch.where(a > 0, a, 1.0)[:, None]), 0.0), a


def within(out, ref, bound, what=""):
    out, ref = out.double(), ref.double()
    assert out.shape == ref.shape, (what, out.shape, ref.shape)
    bad = ~((out - ref).abs() <= bound)
    assert not bad.any(), "%s: %d of %d outside, first at %s: %r, wanted %r" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), out[bad][0].item(), ref[bad][0].item())
