"""Selection, expert order and balance loss behind the router, against their definitions in 64 bits."""
import pytest
import torch

import operator_reference as R
import paper_2607_22595_b200 as mix

pytestmark = pytest.mark.gpu
DEV = "cuda"
ACT = {"softmax": mix.MIX_ACT_SOFTMAX, "sigmoid": mix.MIX_ACT_SIGMOID}
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _logits(T, E, dtype, seed, special=True, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn((T, E), generator=g)
    if special and T >= 8:
        x[1] = -torch.inf                                  # nothing is left of this row
        x[2, E // 2:] = -torch.inf                         # fewer experts than k, maybe
        x[3, E // 3] = torch.inf                           # forced in
        x[4, ::2] = torch.inf                              # more forced in than k, maybe
        x[5, 0] = torch.nan
        x[6] = torch.round(x[6])                           # ties
        x[7] = 0.0
        if T >= 16:
            x[8] = -200.0 + x[8]                           # every sigmoid underflows
            x[9] = 60.0 + x[9]
            x[10] = torch.finfo(DTYPES[dtype]).min         # masks of the type's lowest value
            x[11, 0] = torch.finfo(DTYPES[dtype]).min
            x[12] = -torch.inf
            x[12, E - 1] = 1.0
    return x.to(DTYPES[dtype]).to(DEV)


SIZES = [(1, 1, 1), (1, 8, 2), (3, 2, 2), (17, 7, 3), (64, 8, 8), (33, 9, 2), (40, 16, 16), (29, 31, 4), (70, 33, 6), (64, 64, 8), (31, 100, 16),
         (19, 160, 6), (50, 256, 8), (20, 257, 8), (24, 512, 16), (300, 64, 6)]


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("act,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_topk_and_its_gradient(T, E, k, dtype, act, renorm):
    x = _logits(T, E, dtype, seed=T * 1000 + E)
    idx, w = mix.router_topk(x, k, act=ACT[act], renormalise=renorm)
    ref_idx, ref_w = R.topk(x, k, act, renorm)
    assert torch.equal(idx.cpu().long(), ref_idx)
    # rows of the type's lowest value reach far, but their logits are equal or that one's exponential is 0: no exponent is off
    ordinary = torch.ones(T, dtype=torch.bool)
    ordinary[10:12] = T < 16
    rel = R.rel_p(x[ordinary.to(DEV)], act)
    R.within(w.cpu(), ref_w, rel * ref_w + 1e-37, "weights")
    g = torch.Generator().manual_seed(7)
    d_w = torch.randn((T, k), generator=g)
    d_w[ref_idx < 0] = torch.nan                           # entries without an expert do not count
    d = mix.router_topk_grad(x, idx, w, d_w.to(DEV), act=ACT[act], renormalise=renorm)
    ref, size = R.topk_grad(x.cpu().double(), ref_idx, act, renorm, torch.nan_to_num(d_w))
    R.within(d.cpu(), ref, (2 * rel + 24 * R.U) * size + R.rounding(x.dtype, ref), "d_logits")


@pytest.mark.parametrize("act,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_topk_gradient_against_differences(act, renorm):
    T, E, k = 40, 24, 4
    x = _logits(T, E, "fp32", seed=5, special=False)
    idx, w = mix.router_topk(x, k, act=ACT[act], renormalise=renorm)
    g = torch.Generator().manual_seed(8)
    d_w, along = torch.randn((T, k), generator=g), torch.randn((T, E), generator=g, dtype=torch.float64)
    d = mix.router_topk_grad(x, idx, w, d_w.to(DEV), act=ACT[act], renormalise=renorm).cpu().double()
    x64, i64, h = x.cpu().double(), idx.cpu().long(), 1e-5
    f = lambda y: (R.weights_of(y, i64, act, renorm) * d_w.double()).sum(1)
    change = (f(x64 + h * along) - f(x64 - h * along)) / (2 * h)
    # the kernel's own error as above; of the differences: h^2 / 6 times a third derivative of at most 6 |d_w| (sum |along|)^3, some
    # 1e-10 * 6 * 4 * 20^3 / 6 = 3e-6, and 2^-53 |f| / h
    _, size = R.topk_grad(x64, i64, act, renorm, d_w)
    own = ((2 * R.rel_p(x, act) + 25 * R.U) * size * along.abs()).sum(1)
    R.within((d * along).sum(1), change, own + 1e-10 * d_w.abs().sum(1) * along.abs().sum(1) ** 3, "directional derivative")


def test_rows_behind_the_live_ones_are_not_read_and_get_no_expert():
    x = _logits(50, 32, "fp32", seed=3)
    want_i, want_w = mix.router_topk(x, 4)
    x[33:] = torch.nan
    for live in (0, 1, 33, 50, 99, -5):
        n = torch.tensor([live], dtype=torch.int32, device=DEV)
        idx, w = mix.router_topk(x if live <= 33 else _logits(50, 32, "fp32", seed=3), 4, n_live=n)
        at = min(max(live, 0), 50)
        assert torch.equal(idx[:at], want_i[:at]) and torch.equal(w[:at], want_w[:at])
        assert (idx[at:] == -1).all() and (w[at:] == 0).all()


@pytest.mark.parametrize("dtype,E,pad,shift", [("fp32", 64, 3, 0), ("bf16", 64, 1, 0), ("bf16", 64, 8, 3), ("fp16", 40, 0, 1), ("fp32", 250, 6, 2)])
def test_strides_and_alignments(dtype, E, pad, shift):
    T, k = 37, 5
    base = torch.full((T * (E + pad) + shift,), torch.nan, dtype=DTYPES[dtype], device=DEV)
    x = base[shift:].view(T, E + pad)[:, :E]
    x.copy_(_logits(T, E, dtype, seed=11))
    dense = x.contiguous().clone()
    idx, w = mix.router_topk(x, k, renormalise=False)
    want_i, want_w = mix.router_topk(dense, k, renormalise=False)
    assert torch.equal(idx, want_i) and torch.equal(w, want_w)
    d_w = torch.randn((T, k), device=DEV)
    out = torch.full_like(base, 7.0)
    view = out[shift:].view(T, E + pad)[:, :E]
    assert mix.router_topk_grad(x, idx, w, d_w, renormalise=False, d_logits=view) is view
    assert torch.equal(view, mix.router_topk_grad(dense, idx, w, d_w, renormalise=False))
    assert (out[:shift] == 7).all() and (out[shift:].view(T, E + pad)[:, E:] == 7).all()
    for a, b in zip(mix.router_balance(x, idx), mix.router_balance(dense, idx)):
        assert torch.equal(a, b)
    _, counts, _, rows = mix.router_balance(x, idx)
    one = torch.ones(1, device=DEV)
    out.fill_(7.0)
    mix.router_balance_grad(x, idx, counts, rows, one, d_logits=view)
    assert torch.equal(view, mix.router_balance_grad(dense, idx, counts, rows, one))
    assert (out[:shift] == 7).all() and (out[shift:].view(T, E + pad)[:, E:] == 7).all()


def test_the_same_expert_twice_in_a_row():
    x = _logits(9, 8, "fp32", seed=2, special=False)
    idx = torch.tensor([[3, 3]] * 9, dtype=torch.int32, device=DEV)
    w, d_w = torch.rand((9, 2), device=DEV), torch.randn((9, 2), device=DEV)
    d = mix.router_topk_grad(x, idx, w, d_w, renormalise=True).cpu().double()
    w, g = w.cpu().double(), d_w.cpu().double()
    part = w * (g - (w * g).sum(1, keepdim=True))
    R.within(d[:, 3], part.sum(1), 16 * R.U * (w * (g.abs() + (w * g).abs().sum(1, keepdim=True))).sum(1))
    assert (d[:, :3] == 0).all() and (d[:, 4:] == 0).all()
    loss, counts, mean_p, rows = mix.router_balance(x, idx)
    assert counts[0].tolist() == [0, 0, 0, 18, 0, 0, 0, 0] and rows.tolist() == [9]


ORDERS = [(0, 2, 8), (1, 1, 1), (1, 2, 8), (64, 2, 8), (100, 6, 64), (511, 8, 33), (512, 8, 256), (513, 8, 512), (1000, 5, 7), (3000, 8, 100), (4096, 2, 9), (4097, 2, 3), (5000, 16, 511), (4096, 16, 64), (4097, 16, 64), (20000, 6, 100), (1024, 1, 5), (1025, 1, 5), (2050, 1, 300), (8192, 2, 8), (8193, 2, 8), (41000, 8, 12), (90000, 8, 7), (100000, 14, 4)]


@pytest.mark.parametrize("T,k,E", ORDERS)
def test_expert_order(T, k, E):
    g = torch.Generator().manual_seed(T + E)
    idx = torch.randint(0, E, (T, k), generator=g, dtype=torch.int32)
    idx[torch.rand((T, k), generator=g) < 0.1] = -1
    if T > 60:
        idx[50] = E                                        # no expert either
        idx[51] = 2**31 - 1
        idx[52] = -2**31
    out = mix.expert_order(idx.to(DEV), E)
    for got, want, name in zip(out, R.order(idx, E), ("offsets", "order", "position")):
        assert got.cpu().reshape(-1).tolist() == want, name


def test_expert_order_of_one_expert_and_of_none():
    for fill, counts in ((5, 9000), (-1, 0)):
        idx = torch.full((4500, 2), fill, dtype=torch.int32, device=DEV)
        offsets, order, position = mix.expert_order(idx, 12)
        assert offsets.tolist() == [0] * 6 + [counts] * 7
        there = torch.arange(9000, device=DEV, dtype=torch.int32)
        assert torch.equal(order, there if counts else torch.full_like(there, -1))
        assert torch.equal(position.view(-1), order)


def _segments(kind, T):
    return {"one": None, "two": [0, T // 3, T], "ragged": sorted({0, 1, T // 7, T // 2, T // 2 + 1, T - T // 5}),
            "empty": [0, 0, T // 2, T // 2, T // 2, T, T], "rows": list(range(T + 1)), "inner": [min(5, T), min(9, T), T - T // 4],
            "none": [0, 0]}[kind]


@pytest.mark.parametrize("kind", ["one", "two", "ragged", "empty", "rows", "inner", "none"])
@pytest.mark.parametrize("T,E,k", [(1, 8, 2), (40, 8, 2), (77, 9, 3), (200, 33, 4), (130, 100, 6), (300, 256, 8), (90, 400, 8), (2500, 16, 2), (900, 64, 6)])
@pytest.mark.parametrize("dtype,act", [("fp32", "softmax"), ("bf16", "softmax"), ("fp16", "sigmoid"), ("fp32", "sigmoid")])
def test_balance_and_its_gradient(kind, T, E, k, dtype, act):
    if kind == "rows" and T > 300:
        T = 300
    x = _logits(T, E, dtype, seed=T + E)
    ordinary = torch.ones(T, dtype=torch.bool)
    ordinary[10:12] = T < 16
    idx, _ = mix.router_topk(x, k, act=ACT[act])
    if T > 20:
        idx[17] = -1
        idx[18, 0] = E                                     # no expert
    seg = _segments(kind, T)
    seg_dev = None if seg is None else torch.tensor(seg, dtype=torch.int32, device=DEV)
    listed = [0, T] if seg is None else seg
    loss, counts, mean_p, rows = mix.router_balance(x, idx, seg_dev, act=ACT[act])
    x64, i64 = x.cpu().double(), idx.cpu().long()
    r_loss, r_counts, r_mean, r_rows = R.balance(x64, i64, listed, act)
    assert torch.equal(counts.cpu().long(), r_counts) and rows.tolist() == r_rows
    # every term of the sums is positive, so their relative error is that of a term, U an addition (at most 64 of them one
    # after the other) and the rounding at the end
    rel = R.rel_p(x[ordinary.to(DEV)], act) + 72 * R.U
    R.within(mean_p.cpu(), r_mean, rel * r_mean + 1e-37, "mean_p")
    R.within(loss.cpu(), r_loss, rel * r_loss + 1e-37, "loss")
    d_loss = torch.randn(len(listed) - 1, generator=torch.Generator().manual_seed(1))
    d = mix.router_balance_grad(x, idx, counts, rows, d_loss.to(DEV), seg_dev, act=ACT[act])
    ref, size = R.balance_grad(x64, i64, listed, act, d_loss)
    R.within(d.cpu(), ref, (2 * rel + 24 * R.U) * size + R.rounding(x.dtype, ref), "d_logits")


@pytest.mark.parametrize("act", ["softmax", "sigmoid"])
def test_balance_gradient_against_differences(act):
    T, E, k = 60, 20, 3
    x = _logits(T, E, "fp32", seed=9, special=False)
    idx, _ = mix.router_topk(x, k, act=ACT[act])
    seg = [0, 11, 11, 50]
    seg_dev = torch.tensor(seg, dtype=torch.int32, device=DEV)
    _, counts, _, rows = mix.router_balance(x, idx, seg_dev, act=ACT[act])
    g = torch.Generator().manual_seed(4)
    d_loss, along = torch.randn(3, generator=g), torch.randn((T, E), generator=g, dtype=torch.float64)
    d = mix.router_balance_grad(x, idx, counts, rows, d_loss.to(DEV), seg_dev, act=ACT[act]).cpu().double()
    assert (d[50:] == 0).all()
    f = lambda y: (R.balance(y, idx.cpu().long(), seg, act)[0] * d_loss.double()).sum()
    h = 1e-5
    change = (f(x.cpu().double() + h * along) - f(x.cpu().double() - h * along)) / (2 * h)
    # the kernel's own error as above; of the differences: 2^-53 E / h = 2e-10 and h^2 / 6 times a third derivative, which for a
    # row is at most 6 E / n (sum |along|)^3
    _, size = R.balance_grad(x.cpu().double(), idx.cpu().long(), seg, act, d_loss)
    own = ((2 * R.rel_p(x, act) + 25 * R.U) * size * along.abs()).sum()
    R.within((d * along).sum(), change, own + 1e-9 + 1e-10 * E / 11 * (along.abs().sum(1) ** 3 * d_loss.abs().max()).sum())


def test_balance_of_a_long_batch_gives_the_same_bits_every_time():
    T, E, k = 40000, 96, 4
    x = _logits(T, E, "bf16", seed=12)
    idx, _ = mix.router_topk(x, k)
    seg = torch.tensor([0, 9000, 39990], dtype=torch.int32, device=DEV)
    first = mix.router_balance(x, idx, seg)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, mix.router_balance(x, idx, seg)))
    r_loss, r_counts, r_mean, r_rows = R.balance(x.double(), idx.long(), [0, 9000, 39990], "softmax")
    assert torch.equal(first[1].long(), r_counts) and first[3].tolist() == r_rows
    ordinary = torch.ones(T, dtype=torch.bool, device=DEV)
    ordinary[10:12] = False
    rel = R.rel_p(x[ordinary], "softmax") + 72 * R.U
    R.within(first[2], r_mean, rel * r_mean)
    R.within(first[0], r_loss, rel * r_loss)


def test_captured_with_rewritten_inputs_and_on_another_stream():
    T, E, k = 700, 64, 6
    x = _logits(T, E, "bf16", seed=21)
    n_live = torch.tensor([650], dtype=torch.int32, device=DEV)
    seg = torch.tensor([0, 300, 650], dtype=torch.int32, device=DEV)
    d_w, d_loss = torch.randn((T, k), device=DEV), torch.randn(2, device=DEV)

    def step():
        idx, w = mix.router_topk(x, k, n_live=n_live)
        loss, counts, mean_p, rows = mix.router_balance(x, idx, seg)
        return (idx, w, *mix.expert_order(idx, E), mix.router_topk_grad(x, idx, w, d_w), loss, counts, mean_p, rows,
                mix.router_balance_grad(x, idx, counts, rows, d_loss, seg))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm = step()
    torch.cuda.current_stream().wait_stream(side)
    want = step()
    assert all(torch.equal(a, b) for a, b in zip(warm, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed, live, cut in ((22, 650, 300), (23, 400, 10), (24, 0, 0)):
        x.copy_(_logits(T, E, "bf16", seed=seed))
        n_live.fill_(live)
        seg.copy_(torch.tensor([0, cut, live], dtype=torch.int32))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, step()))


def test_expert_order_of_many_entries():
    """More entries than the host sorts in reasonable time: against a stable sort."""
    for T, k, E in ((300000, 8, 512), (1 << 20, 16, 3)):
        g = torch.Generator(device=DEV).manual_seed(E)
        idx = torch.randint(-1, E, (T, k), generator=g, device=DEV, dtype=torch.int32)
        offsets, order, position = mix.expert_order(idx, E)
        key = torch.where(idx.view(-1) < 0, E, idx.view(-1)).long()
        want = torch.sort(key, stable=True).indices
        counts = torch.bincount(key, minlength=E + 1)
        assert torch.equal(offsets.long(), torch.cat([torch.zeros_like(counts[:1]), counts[:E].cumsum(0)]))
        n = int(offsets[-1])
        assert torch.equal(order[:n].long(), want[:n]) and (order[n:] == -1).all()
        place = torch.empty_like(want)
        place[want] = torch.arange(T * k, device=DEV)
        assert torch.equal(position.view(-1).long(), torch.where(key < E, place, -1))


def test_no_rows():
    x, none = torch.empty((0, 12), device=DEV), torch.empty((0, 3), dtype=torch.int32, device=DEV)
    idx, w = mix.router_topk(x, 3)
    assert idx.shape == (0, 3) and w.shape == (0, 3)
    assert mix.router_topk_grad(x, idx, w, w).shape == (0, 12)
    for seg in (None, torch.zeros(5, dtype=torch.int32, device=DEV)):
        loss, counts, mean_p, rows = mix.router_balance(x, none, seg)
        n = 1 if seg is None else 4
        assert loss.shape == (n,) and not loss.any() and counts.shape == (n, 12) and not counts.any() and not mean_p.any() and not rows.any()
        assert mix.router_balance_grad(x, none, counts, rows, torch.ones(n, device=DEV), seg).shape == (0, 12)


def test_outputs_that_are_given_and_refused():
    x = _logits(20, 16, "fp32", seed=1)
    idx, w = torch.empty((20, 4), dtype=torch.int32, device=DEV), torch.empty((20, 4), device=DEV)
    out = mix.router_topk(x, 4, idx=idx, weights=w)
    assert out[0] is idx and out[1] is w
    offsets, order, position = (torch.empty(s, dtype=torch.int32, device=DEV) for s in ((17,), (80,), (20, 4)))
    got = mix.expert_order(idx, 16, offsets=offsets, order=order, position=position)
    assert got[0] is offsets and got[1] is order and got[2] is position and offsets[-1] == (idx >= 0).sum()
    long = idx.long()
    for call in (lambda: mix.router_topk(x, 0), lambda: mix.router_topk(x, 17), lambda: mix.router_topk(x, 4, idx=idx[:, :3], weights=w),
                 lambda: mix.router_topk(x, 4, idx=long, weights=w), lambda: mix.router_topk(x.double(), 4), lambda: mix.router_topk(x[0], 4),
                 lambda: mix.router_topk(x.t(), 4), lambda: mix.router_topk(x, 4, n_live=torch.ones(2, dtype=torch.int32, device=DEV)),
                 lambda: mix.router_topk(x, 4, act=7), lambda: mix.expert_order(long, 16), lambda: mix.expert_order(idx, 0),
                 lambda: mix.expert_order(idx.t(), 16), lambda: mix.router_topk_grad(x, idx, w, w.double()),
                 lambda: mix.router_topk_grad(x, idx, w, w, d_logits=torch.empty_like(x, dtype=torch.bfloat16)),
                 lambda: mix.router_balance(x, long), lambda: mix.router_balance(x, idx, torch.zeros(1, dtype=torch.int32, device=DEV)),
                 lambda: mix.router_balance(x, idx, torch.zeros(3, device=DEV)), lambda: mix.router_balance(x[:19], idx)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(mix.MixError) as e:
        mix.router_topk(torch.zeros((4, 600), device=DEV), 2)
    assert e.value.code == -2 and "n_experts" in str(e.value)
    with pytest.raises(mix.MixError):
        mix.router_topk(x[:1].expand(20, 16), 4)           # rows that lie on top of each other
    with pytest.raises(mix.MixError):
        mix.router_topk(x, 4, act=mix.MIX_ACT_NONE)


@pytest.mark.parametrize("act", ["softmax", "sigmoid"])
def test_a_single_chosen_expert_has_weight_one_and_no_gradient(act):
    for E in (1, 5, 64, 100, 300):
        x = _logits(200, E, "fp32", seed=E, special=False, spread=4.0)
        idx, w = mix.router_topk(x, 1, act=ACT[act])
        assert (w == 1).all()
        assert not mix.router_topk_grad(x, idx, w, torch.randn((200, 1), device=DEV), act=ACT[act]).any()


def test_balance_gradient_is_zero_where_all_experts_are_chosen_alike():
    for T, E in ((1, 2), (30, 3), (400, 7), (50, 16)):
        x = _logits(T, E, "fp32", seed=E, special=False)
        idx = torch.arange(E, dtype=torch.int32, device=DEV).repeat(T, 1)
        for act in ("softmax", "sigmoid"):
            loss, counts, mean_p, rows = mix.router_balance(x, idx, act=ACT[act])
            R.within(loss, torch.ones_like(loss), (R.rel_p(x, act) + 72 * R.U) * torch.ones(1, device=DEV))
            assert not mix.router_balance_grad(x, idx, counts, rows, loss, act=ACT[act]).any()


def test_balance_gradient_of_nearly_even_shares():
    """All but one of eight experts chosen: what is left of the shares is small, and still right to fp32's precision."""
    x = _logits(1, 8, "fp32", seed=3, special=False, spread=3.0)
    idx, _ = mix.router_topk(x, 7)
    loss, counts, _, rows = mix.router_balance(x, idx)
    one = torch.ones(1)
    d = mix.router_balance_grad(x, idx, counts, rows, one.to(DEV))
    ref, _ = R.balance_grad(x.cpu().double(), idx.cpu().long(), [0, 1], "softmax", one)
    # f_j - f_max is 0 or -1 / 7, each entry a product of two probabilities (or p (1 - p)), with the same relative bound twice
    p = R.probabilities(x.cpu().double(), "softmax")
    out = p.argmin()
    terms = p * p[0, out]
    terms[0, out] = p[0, out] * (1 + p[0, out])
    R.within(d.cpu(), ref, (2 * R.rel_p(x, "softmax") + 24 * R.U) * 8 / 7 * terms)


@pytest.mark.parametrize("E", [3, 8, 9, 16, 17, 33, 64, 65, 80, 128, 129, 200, 256, 300, 512])
def test_logits_that_differ_in_their_last_bits(E):
    """fp32 logits a few steps apart, chosen and not chosen ones among them, below and above 0, at every k."""
    T = 400
    g = torch.Generator().manual_seed(E)
    steps = torch.stack([torch.randperm(4 * E, generator=g)[:E] for _ in range(T)]).double()
    x = (1.0 + steps * 2.0**-23) * torch.where(torch.rand((T, 1), generator=g) < 0.5, -1.0, 1.0).double()
    few = torch.rand((T, E), generator=g) < 0.7               # in half of the rows only a few are close to each other
    x = torch.where(few & (torch.arange(T)[:, None] % 2 == 0), x * 2.0 ** torch.randint(-3, 3, (T, E), generator=g), x).float()
    want = torch.sort(x.double(), dim=1, descending=True, stable=True).indices
    for k in sorted({1, 2, min(8, E), min(15, E), min(16, E)}):
        idx, _ = mix.router_topk(x.to(DEV), k)
        assert torch.equal(idx.cpu().long(), want[:, :k]), k
