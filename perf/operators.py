"""Performance cases of the router operators and of the products in 8-bit integers.

Four operators through the public entry points:

  route    the experts of each token from its router logits, their weights, and the tokens sorted by expert:
           `router_topk`, `expert_order`; in training also the gradient of the weights: `router_topk_grad`
  balance  how evenly the router spreads each request's tokens: per-expert counts, mean probabilities and the balance
           loss, `router_balance`, and the loss's gradient, `router_balance_grad`
  linear   y = x W^T with x quantised to 8-bit integers per token and W held in 8-bit integers with a scale per output
           channel: `quantize_rows`, `linear_int`
  experts  the same product where each token goes through the experts that its router chose: `expert_order`,
           `quantize_rows` in the order of the experts, `linear_int_grouped`, and, where a token's results are summed
           again, `expert_combine`
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


# ------------------------------------------------------------------------------------------ the cases
def _route(name, T, E, k, live, dtype="fp32", act="softmax", renorm=True, train=False):
    """live: tokens of the step; the rows behind them, up to T, are padding."""
    c = dict(op="route", T=T, E=E, k=k, live=live, dtype=dtype, act=act, renorm=renorm, train=train)
    return dict(name=name, **c) if name else c


def _balance(name, T, E, k, requests, live, dtype="fp32", act="softmax"):
    """requests: segments of the loss, of ragged lengths that add up to `live`."""
    c = dict(op="balance", T=T, E=E, k=k, requests=requests, live=live, dtype=dtype, act=act)
    return dict(name=name, **c) if name else c


def _linear(name, T, K, N, dtype="bf16", bias=False):
    c = dict(op="linear", T=T, K=K, N=N, dtype=dtype, bias=bias)
    return dict(name=name, **c) if name else c


def _experts(name, T, E, k, K, N, live, skew=0.5, dtype="bf16", combine=False):
    """skew: spread of the experts' popularity (0: all alike)."""
    c = dict(op="experts", T=T, E=E, k=k, K=K, N=N, live=live, skew=skew, dtype=dtype, combine=combine)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # a decode step of 64 requests on eight experts, two a token: nothing but latency
        _route("route_decode", T=64, E=8, k=2, live=64),
        # a mixed step of prefill and decode tokens at the large capture size, logits in the model's type, the last rows padding
        _route("route_mixed_step", T=8192, E=64, k=6, live=7777, dtype="bf16"),
        # a training batch on many small experts, weights as the probabilities are, with the gradient
        _route("route_train", T=65536, E=256, k=8, live=65536, renorm=False, train=True),
        # the load of one odd-sized batch
        _balance("balance_one_batch", T=517, E=8, k=2, requests=1, live=517),
        # ragged requests of a mixed step: which experts each request's tokens went to, and a loss a request
        _balance("balance_64_requests", T=8192, E=64, k=6, requests=64, live=7777, dtype="bf16"),
        # a training batch of 16 long sequences, scores by sigmoid
        _balance("balance_train", T=65536, E=256, k=8, requests=16, live=65536, act="sigmoid"),
        # a decode step of 16 requests: the stream of the weights
        _linear("linear_decode", T=16, K=4096, N=16384),
        # a prefill chunk of odd sizes, with a bias
        _linear("linear_chunk", T=1000, K=5120, N=9992, dtype="fp16", bias=True),
        # the mixed step's largest product
        _linear("linear_prefill", T=8192, K=8192, N=32768),
        # a decode step of 64 requests: the weights of all eight experts for sixteen rows each
        _experts("experts_decode", T=64, E=8, k=2, K=4096, N=8192, live=64),
        # the way back of many small experts, summed over each token's experts, the last rows padding
        _experts("experts_down", T=2048, E=64, k=6, K=2048, N=5120, live=1999, combine=True),
        # a prefill batch on eight large experts
        _experts("experts_prefill", T=8192, E=8, k=2, K=4096, N=16384, live=8192, skew=0.7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _live(rng, T):
    return T if rng.random() < 0.5 else rng.randint(max(1, T // 2), T)


def draw(rng):
    op = rng.choice(["route", "balance", "linear", "experts"])
    if op in ("route", "balance"):
        E = rng.choice([rng.randint(2, 32), _log(rng, 8, 320), rng.choice([8, 16, 32, 64, 128, 160, 256])])
        k = rng.randint(1, min(8, E))
        T = _log(rng, 1, min(65536, 65536 * 256 // max(E, 64)))
        dtype, act = rng.choice(["fp32", "fp32", "bf16", "fp16"]), rng.choice(["softmax", "softmax", "sigmoid"])
        if op == "route":
            return _route(None, T, E, k, _live(rng, T), dtype, act, rng.random() < 0.6, rng.random() < 0.5)
        return _balance(None, T, E, k, _log(rng, 1, max(1, min(T, 256))), _live(rng, T), dtype, act)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op == "linear":
        T, K = _log(rng, 1, 8192), 16 * _log(rng, 8, 512)
        N = rng.choice([_log(rng, 64, 32768), 128 * _log(rng, 1, 256)])
        return _linear(None, T, K, N, dtype, rng.random() < 0.4)
    E = rng.choice([rng.randint(2, 32), 8, 16, 64])
    k = rng.randint(1, min(8, E))
    K, N = 16 * _log(rng, 16, 256), rng.choice([_log(rng, 256, 8192), 128 * _log(rng, 2, 64)])
    T = _log(rng, 1, 16384 // k)
    return _experts(None, T, E, k, K, N, _live(rng, T), rng.choice([0.0, 0.5, 1.5]), dtype, rng.random() < 0.5)


# ------------------------------------------------------------------------------------------ the inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _logits(g, T, E, dtype, skew=0.7):
    """Router logits: some experts are more popular than others; in a tenth of the rows a steering app has forced one
    expert out, in a hundredth another one in."""
    x = 1.5 * torch.randn((T, E), generator=g, device="cuda") + skew * torch.randn((1, E), generator=g, device="cuda")
    who = torch.rand((T, 1), generator=g, device="cuda")
    out, into = torch.randint(0, E, (2,), generator=g, device="cuda")
    at = torch.arange(E, device="cuda")[None]
    x = torch.where((who < 0.1) & (at == out), -math.inf, x)
    x = torch.where((who > 0.99) & (at == into), math.inf, x)
    return x.to(DTYPES[dtype])


def _chosen(x, k, live):
    idx = torch.topk(x.float(), k, dim=1).indices.to(torch.int32)
    idx[live:] = -1
    return idx.contiguous()


def _segments(g, n, live):
    """Offsets of n ragged segments that cover the live rows; where there are many, one of them is empty."""
    w = torch.exp(torch.randn(n, generator=g, device="cuda", dtype=torch.float64))
    if n > 4:
        w[n // 2] = 0
    end = torch.floor(torch.cumsum(w, 0) / w.sum() * live + 0.5).to(torch.int32)
    end[-1] = live
    return torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), end]).contiguous()


def _activations(g, T, K, dtype):
    """Hidden states: a few channels are much larger than the rest."""
    x = torch.randn((T, K), generator=g, device="cuda")
    x *= torch.where(torch.rand((1, K), generator=g, device="cuda") < 0.01, 8.0, 1.0)
    return x.to(DTYPES[dtype])


def _weights_i8(g, shape):
    w = torch.empty(shape, dtype=torch.int8, device="cuda")
    flat = w.view(-1, shape[-1])
    for i in range(0, flat.shape[0], 8192):          # normal values of which the largest of a channel is about 127
        part = flat[i:i + 8192]
        part.copy_((32 * torch.randn(part.shape, generator=g, device="cuda")).round().clamp(-127, 127))
    scale = (0.5 + torch.rand(shape[:-1], generator=g, device="cuda")) / (32 * math.sqrt(shape[-1]))
    return w, scale


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case)
    if case["op"] == "route":
        s["logits"] = _logits(g, case["T"], case["E"], case["dtype"])
        s["n_live"] = torch.full((1,), case["live"], dtype=torch.int32, device="cuda")
        s["d_weights"] = torch.randn((case["T"], case["k"]), generator=g, device="cuda")
    elif case["op"] == "balance":
        s["logits"] = _logits(g, case["T"], case["E"], case["dtype"])
        s["idx"] = _chosen(s["logits"], case["k"], case["live"])
        s["seg"] = _segments(g, case["requests"], case["live"])
        s["d_loss"] = 0.5 + torch.rand(case["requests"], generator=g, device="cuda")
    else:
        s["x"] = _activations(g, case["T"], case["K"], case["dtype"])
        if case["op"] == "linear":
            s["w"], s["w_scale"] = _weights_i8(g, (case["N"], case["K"]))
            s["bias"] = torch.randn(case["N"], generator=g, device="cuda") if case["bias"] else None
        else:
            s["w"], s["w_scale"] = _weights_i8(g, (case["E"], case["N"], case["K"]))
            logits = _logits(g, case["T"], case["E"], "fp32", case["skew"])
            # only a sum over the experts has a place for a token without any: elsewhere every row is live
            live = case["live"] if case["combine"] else case["T"]
            s["idx"] = _chosen(logits, case["k"], live)
            s["weights"] = torch.softmax(torch.randn(s["idx"].shape, generator=g, device="cuda"), 1)
            s["weights"][live:] = 0
    if own:
        import paper_2607_22595_b200 as mix
        s["mix"] = mix
        s["act_id"] = mix.MIX_ACT_SIGMOID if case.get("act") == "sigmoid" else mix.MIX_ACT_SOFTMAX
    return s


# ------------------------------------------------------------------------------------------ the passes
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    mix = s["mix"]
    if s["op"] == "route":
        idx, weights = mix.router_topk(s["logits"], s["k"], act=s["act_id"], renormalise=s["renorm"], n_live=s["n_live"])
        offsets, order, position = mix.expert_order(idx, s["E"])
        out = [idx, weights, offsets, order, position]
        if s["train"]:
            out.append(mix.router_topk_grad(s["logits"], idx, weights, s["d_weights"], act=s["act_id"], renormalise=s["renorm"]))
        return out
    if s["op"] == "balance":
        loss, counts, mean_p, rows = mix.router_balance(s["logits"], s["idx"], s["seg"], act=s["act_id"])
        grad = mix.router_balance_grad(s["logits"], s["idx"], counts, rows, s["d_loss"], s["seg"], act=s["act_id"])
        return [loss, counts, mean_p, rows, grad]
    if s["op"] == "linear":
        codes, scale = mix.quantize_rows(s["x"])
        return mix.linear_int(codes, scale, s["w"], s["w_scale"], bias=s["bias"], dtype=s["x"].dtype)
    offsets, order, position = mix.expert_order(s["idx"], s["E"])
    codes, scale = mix.quantize_rows(s["x"], order=order, k=s["k"])
    y = mix.linear_int_grouped(codes, scale, s["w"], s["w_scale"], offsets, dtype=s["x"].dtype)
    return mix.expert_combine(y, s["weights"], position) if s["combine"] else y


# -- the plain forms
def _scores(x, act):
    """Probabilities of the experts, rows of x in 32 bits: NaN counts as -inf, the largest logits share a row of +inf."""
    x = torch.where(torch.isnan(x), -math.inf, x)
    m = x.max(1, keepdim=True).values
    if act == "softmax":
        e = torch.where(x == m, torch.ones_like(x), torch.exp(x - m))
        e = torch.where(x == -math.inf, torch.zeros_like(e), e)
    else:
        c = m.clamp(max=0.0)                          # sigmoid(x) e^-c: nothing underflows where all logits are low
        e = torch.where(x > 0, torch.exp(-c) / (1 + torch.exp(-x)), torch.exp(x - c) / (1 + torch.exp(x)))
        e = torch.where(x == -math.inf, torch.zeros_like(e), e)
    return e


def _share(e):
    total = e.sum(1, keepdim=True)
    return torch.where(total > 0, e / total, torch.zeros_like(e))


def _order(idx, E):
    flat = idx.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = torch.sort(key, stable=True).indices
    counts = torch.zeros(E + 1, dtype=torch.long, device=key.device).scatter_add_(0, key, torch.ones_like(key))[:E]
    offsets = torch.cat([torch.zeros(1, dtype=torch.long, device=key.device), torch.cumsum(counts, 0)])
    place = torch.arange(key.numel(), device=key.device)
    position = torch.empty_like(place)
    position[order] = place
    position = torch.where(flat < 0, -1, position)
    order = torch.where(place < offsets[-1], order, -1)
    return offsets.int(), order.int(), position.int().view(idx.shape)


def _run_plain(s):
    if s["op"] == "route":
        return _plain_route(s)
    if s["op"] == "balance":
        return _plain_balance(s)
    if s["op"] == "linear":
        codes, scale = _quantized(s["x"])
        y = _product(codes, s["w"]) * scale[:, None] * s["w_scale"][None]
        if s["bias"] is not None:
            y = y + s["bias"][None]
        return y.to(s["x"].dtype)
    return _plain_experts(s)


def _plain_route(s):
    T, E, k = s["T"], s["E"], s["k"]
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    value, idx = torch.sort(x, dim=1, descending=True, stable=True)
    value, idx = value[:, :k], idx[:, :k]
    there = (value > -math.inf) & (torch.arange(T, device=x.device) < s["n_live"])[:, None]
    if s["act"] == "softmax":
        e = _scores(x, "softmax")
        chosen = torch.where(there, e.gather(1, idx), 0.0)
        weights = chosen / (chosen if s["renorm"] else e).sum(1, keepdim=True)
    else:
        e = _scores(x, "sigmoid") if s["renorm"] else 1 / (1 + torch.exp(-x))
        weights = torch.where(there, e.gather(1, idx), 0.0)
        if s["renorm"]:
            weights = weights / weights.sum(1, keepdim=True)
    weights = torch.where(there, weights, 0.0)
    idx = torch.where(there, idx, -1).int()
    out = [idx, weights, *_order(idx, E)]
    if s["train"]:
        g = torch.where(there, s["d_weights"], 0.0)
        at = idx.clamp(min=0).long()
        if s["act"] == "softmax" and not s["renorm"]:
            d = torch.zeros_like(x).scatter_add_(1, at, g)
            p = torch.where(there.any(1, keepdim=True), _share(e), 0.0)
            d = p * (d - (g * weights).sum(1, keepdim=True))
        else:
            if s["act"] == "softmax":
                part = weights * (g - (g * weights).sum(1, keepdim=True))
            else:
                rest = 1 / (1 + torch.exp(x.gather(1, at)))
                part = weights * rest * (g - (g * weights).sum(1, keepdim=True) if s["renorm"] else g)
            d = torch.zeros_like(x).scatter_add_(1, at, torch.where(there, part, 0.0))
        out.append(d.to(s["logits"].dtype))
    return out


def _plain_balance(s):
    T, E, n = s["T"], s["E"], s["requests"]
    x, idx, seg = s["logits"].float(), s["idx"].long(), s["seg"].long()
    row = torch.arange(T, device=x.device)
    which = (row[:, None] >= seg[None, 1:]).sum(1)                  # the row's request; n behind the last one
    named = (idx >= 0) & (idx < E)
    on = named.any(1) & (which < n)
    which = torch.where(on, which, n)
    e = _scores(x, s["act"])
    p = torch.where(on[:, None], _share(e), 0.0)
    flat = torch.where(named & on[:, None], which[:, None] * E + idx, n * E)
    counts = torch.zeros(n * E + 1, dtype=torch.long, device=x.device).scatter_add_(0, flat.reshape(-1), torch.ones_like(flat).reshape(-1))
    counts = counts[:-1].view(n, E)
    rows = torch.zeros(n + 1, dtype=torch.long, device=x.device).scatter_add_(0, which, torch.ones_like(which))[:n]
    total = torch.zeros((n + 1, E), dtype=torch.float64, device=x.device).index_add_(0, which, p.double())[:n]
    mean_p = total / rows.clamp(min=1)[:, None]
    f = counts.double() / counts.sum(1, keepdim=True).clamp(min=1)
    loss = E * (f * mean_p).sum(1)
    fr = torch.cat([f, torch.zeros_like(f[:1])]).float()[which]
    scale = torch.cat([s["d_loss"] * E / rows.clamp(min=1), torch.zeros_like(s["d_loss"][:1])])[which]
    inner = fr - (fr * p).sum(1, keepdim=True)
    d = scale[:, None] * p * inner
    if s["act"] == "sigmoid":
        d = d / (1 + torch.exp(x))
    d = torch.where(on[:, None] & (x > -math.inf), d, 0.0)
    return [loss.float(), counts.int(), mean_p.float(), rows.int(), d.to(s["logits"].dtype)]


def _quantized(x):
    """Whole numbers from -127 to 127 in 32-bit floats, and the scale of each row."""
    x = x.float()
    a = x.abs().amax(1)
    codes = torch.round(127 * x / torch.where(a > 0, a, 1.0)[:, None])
    return codes, a / 127


def _product(codes, w):
    """codes @ w^T: sums of 1024 products of 8-bit numbers are exact in 32 bits, longer ones are put together from them."""
    y = None
    for i in range(0, codes.shape[1], 1024):
        part = codes[:, i:i + 1024] @ w[:, i:i + 1024].float().t()
        y = part if y is None else y + part
    return y


def _plain_experts(s):
    E, k = s["E"], s["k"]
    offsets, order, position = _order(s["idx"], E)
    codes, scale = _quantized(s["x"])
    y = torch.zeros((order.numel(), s["N"]), device="cuda")
    ends = offsets.tolist()
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        if b > a:
            t = torch.div(order[a:b].long(), k, rounding_mode="floor")
            y[a:b] = _product(codes[t], s["w"][e]) * scale[t][:, None] * s["w_scale"][e][None]
    if not s["combine"]:
        return y.to(s["x"].dtype)
    out = torch.zeros((s["T"], s["N"]), device="cuda")
    for j in range(k):
        at = position[:, j].long()
        out += torch.where(at >= 0, s["weights"][:, j], 0.0)[:, None] * y[at.clamp(min=0)]
    return out.to(s["x"].dtype)


# ------------------------------------------------------------------------------------------ from the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"route": _exact_route, "balance": _exact_balance, "linear": _exact_linear, "experts": _exact_experts}[case["op"]](s)


def _exact_p(x, act):
    """Probabilities in 64 bits. Logits of +inf are the limit of equal ones that grow without bound."""
    top = (x == math.inf)
    high = torch.where(top.any(1, keepdim=True), torch.where(top, 0.0, -math.inf).double(), x)
    if act == "softmax":
        p = torch.softmax(high, 1)
    else:
        logs = torch.nn.functional.logsigmoid(x)
        p = torch.softmax(logs, 1)
    return torch.nan_to_num(p, nan=0.0)


def _exact_route(s):
    x = s["logits"].double()
    T, E, k = s["T"], s["E"], s["k"]
    live = torch.arange(T, device="cuda") < s["live"]
    x = torch.where(torch.isnan(x), -math.inf, x)
    taken = torch.zeros_like(x, dtype=torch.bool)
    picks = []
    for _ in range(k):                                               # the largest, the first of equals, k times
        open_ = torch.where(taken, -math.inf, x)
        best = open_.max(1, keepdim=True).values
        at = ((open_ == best) & ~taken).int().argmax(1)
        ok = (best[:, 0] > -math.inf) & live
        picks.append(torch.where(ok, at, -1))
        taken[torch.arange(T, device="cuda"), at] = True
    idx = torch.stack(picks, 1)
    there = idx >= 0
    at = idx.clamp(min=0)
    mask = torch.zeros_like(x).scatter_add_(1, at, there.double()) > 0
    if s["renorm"]:
        p = _exact_p(torch.where(mask, x, -math.inf), s["act"])
        # the weights of the chosen, as a function of all logits: only the chosen count
        p = torch.where(mask, p, 0.0)
    elif s["act"] == "softmax":
        p = _exact_p(x, "softmax")
    else:
        p = torch.sigmoid(x)
    weights = torch.where(there, p.gather(1, at), 0.0)
    off, order, position = _exact_order(idx, E)
    out = [idx.int(), weights, off, order, position]
    if s["train"]:
        g = torch.zeros_like(x).scatter_add_(1, at, torch.where(there, s["d_weights"].double(), 0.0))
        p = torch.where(live[:, None], p, 0.0)
        if s["act"] == "sigmoid":
            slope = p * torch.sigmoid(-x)
            d = slope * (g - (g * p).sum(1, keepdim=True)) if s["renorm"] else torch.where(mask, slope * g, 0.0)
        else:
            d = p * (g - (g * p).sum(1, keepdim=True))
        out.append(torch.where(p > 0, d, 0.0))
    return out


def _exact_order(idx, E):
    import numpy as np
    flat = idx.reshape(-1).cpu().numpy()
    where = [np.flatnonzero(flat == e) for e in range(E)]
    off = np.concatenate([[0], np.cumsum([len(w) for w in where])])
    order = np.full(flat.size, -1)
    position = np.full(flat.size, -1)
    order[:off[-1]] = np.concatenate(where) if where else []
    position[order[:off[-1]]] = np.arange(off[-1])
    as_i = lambda a: torch.from_numpy(np.ascontiguousarray(a.astype(np.int32))).cuda()
    return as_i(off), as_i(order), as_i(position).view(idx.shape)


def _exact_balance(s):
    x, E = s["logits"].double(), s["E"]
    idx, seg = s["idx"], s["seg"].tolist()
    p = _exact_p(x, s["act"])
    losses, counts, means, ns = [], [], [], []
    d = torch.zeros_like(x)
    for i in range(s["requests"]):
        a, b = seg[i], seg[i + 1]
        rows = (idx[a:b] >= 0).any(1)
        n = int(rows.sum())
        c = torch.stack([(idx[a:b] == e).sum() for e in range(E)]) if E * s["requests"] <= 512 else \
            torch.bincount(idx[a:b][idx[a:b] >= 0].long(), minlength=E)
        pi = p[a:b] * rows[:, None]
        mean = pi.sum(0) / max(n, 1)
        f = c.double() / max(int(c.sum()), 1)
        losses.append(E * (f * mean).sum())
        counts.append(c.int())
        means.append(mean)
        ns.append(n)
        h = s["d_loss"][i].double() * E / max(n, 1) * f
        di = pi * (h[None] - (pi * h[None]).sum(1, keepdim=True))
        d[a:b] = di * torch.sigmoid(-x[a:b]) if s["act"] == "sigmoid" else di
    ns = torch.tensor(ns, dtype=torch.int32, device="cuda")
    return [torch.stack(losses), torch.stack(counts), torch.stack(means), ns, torch.where(p > 0, d, 0.0)]


def _exact_codes(x):
    x = x.double()
    a = x.abs().max(1).values
    return torch.where(a[:, None] > 0, torch.round(x * 127 / a[:, None]), 0.0), a / 127


def _exact_linear(s):
    codes, scale = _exact_codes(s["x"])
    y = torch.empty((s["T"], s["N"]), dtype=torch.float64, device="cuda")
    for i in range(0, s["N"], 4096):
        y[:, i:i + 4096] = torch.mm(codes, s["w"][i:i + 4096].double().t()) * s["w_scale"][i:i + 4096].double() * scale[:, None]
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_experts(s):
    codes, scale = _exact_codes(s["x"])
    idx, k = s["idx"], s["k"]
    out = torch.zeros((s["T"], s["N"]), dtype=torch.float64, device="cuda") if s["combine"] else []
    for e in range(s["E"]):
        t, j = torch.nonzero(idx == e, as_tuple=True)                # by token, then by choice
        y = torch.mm(codes[t], s["w"][e].double().t()) * scale[t][:, None] * s["w_scale"][e].double()
        if s["combine"]:
            out.index_add_(0, t, y * s["weights"][t, j].double()[:, None])
        else:
            out.append(y)
    return out if s["combine"] else torch.cat(out)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    T, E, k = case["T"], case.get("E", 1), case.get("k", 1)
    if case["op"] == "route":
        es = BYTES[case["dtype"]]
        moved = T * E * es + T * k * 8 + T * k * 8 + 4 * (E + 1) + 4
        flops = T * E * 4
        if case["train"]:
            moved += T * k * 4 + T * E * es
            flops += T * E * 4
        return {"bytes": moved, "flops": flops}
    if case["op"] == "balance":
        es = BYTES[case["dtype"]]
        n = case["requests"]
        return {"bytes": 2 * T * E * es + T * k * 4 + n * (8 * E + 12), "flops": T * E * 10}
    K, N, es = case["K"], case["N"], 2
    if case["op"] == "linear":
        return {"bytes": T * K * es + N * K + 4 * N * (2 if case["bias"] else 1) + T * N * es, "flops": 2 * T * N * K}
    rows = (case["live"] if case["combine"] else T) * k
    used = min(E, rows)                                              # experts that can have a row: their weights are read
    moved = T * K * es + used * N * (K + 4) + T * k * 4 + (T * N * es + T * k * 4 if case["combine"] else rows * N * es)
    return {"bytes": moved, "flops": 2 * rows * N * K + (2 * rows * N if case["combine"] else 0)}
