"""Selection, balance loss and their gradients with a bound for each row of logits: rows whose largest logit lies far from 0."""
import pytest
import torch

import operator_reference as R
import paper_2607_22595_b200 as mix

pytestmark = pytest.mark.gpu
DEV = "cuda"
ACT = {"softmax": mix.MIX_ACT_SOFTMAX, "sigmoid": mix.MIX_ACT_SIGMOID}
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def row_bound(x, act):
    """Relative bound on the probabilities of each row [T, 1].  A probability that is not 0 in fp32 is made of e^d, d the logit's distance
    from the row's largest (at most 104), or of e^x where the scores are sigmoids: a power of 2 whose argument is off by 1.22 |d| U (its
    rounding, and log2 e's) and two steps, 4 U.  The difference is exact where the logits are that close to each other and far from
    0.  The sum of the row's terms is off by the mean of that, at most 17 U, and 24 U of additions; reciprocal and products 4 U."""
    x = x.double()
    there = torch.isfinite(x)
    far = _that_count(torch.where(there, torch.where(there, x, -torch.inf).amax(1, keepdim=True) - x, 0.0))
    if act == "sigmoid":
        far = torch.maximum(far, _that_count(torch.where(there, x.abs(), 0.0)))     # each by itself: -40 counts beside 200, though they are 240 apart
    return (2 * (far + 8) + 32) * R.U


def _that_count(d):
    return torch.where(d < 104, d, 0.0).amax(1, keepdim=True)


def check_topk(x, k, act, renorm):
    T = x.shape[0]
    idx, w = mix.router_topk(x, k, act=ACT[act], renormalise=renorm)
    ref_idx, ref_w = R.topk(x, k, act, renorm)
    assert torch.equal(idx.cpu().long(), ref_idx)
    rel = row_bound(x.cpu(), act)
    R.within(w.cpu(), ref_w, rel * ref_w + 1e-37, "weights")
    d_w = torch.randn((T, k), generator=torch.Generator().manual_seed(7))
    d = mix.router_topk_grad(x, idx, w, d_w.to(DEV), act=ACT[act], renormalise=renorm)
    ref, size = R.topk_grad(x.cpu().double(), ref_idx, act, renorm, torch.where(ref_idx >= 0, d_w, 0.0))
    R.within(d.cpu(), ref, (2 * rel + 24 * R.U) * size + R.rounding(x.dtype, ref), "d_logits")


def check_balance(x, k, act, seg, adds=64):
    """adds: probabilities of one expert that are added one after the other in fp32."""
    T = x.shape[0]
    idx, _ = mix.router_topk(x, k, act=ACT[act])
    seg_dev = None if seg is None else torch.tensor(seg, dtype=torch.int32, device=DEV)
    listed = [0, T] if seg is None else seg
    loss, counts, mean_p, rows = mix.router_balance(x, idx, seg_dev, act=ACT[act])
    x64, i64 = x.cpu().double(), idx.cpu().long()
    r_loss, r_counts, r_mean, r_rows = R.balance(x64, i64, listed, act)
    assert torch.equal(counts.cpu().long(), r_counts) and rows.tolist() == r_rows
    rel = row_bound(x.cpu(), act)
    worst = torch.stack([rel[a:b].max() if b > a else rel.new_zeros(()) for a, b in zip(listed[:-1], listed[1:])]) + (adds + 8) * R.U
    R.within(mean_p.cpu(), r_mean, worst[:, None] * r_mean + 1e-37, "mean_p")
    R.within(loss.cpu(), r_loss, worst * r_loss + 1e-37, "loss")
    d_loss = torch.randn(len(listed) - 1, generator=torch.Generator().manual_seed(1))
    d = mix.router_balance_grad(x, idx, counts, rows, d_loss.to(DEV), seg_dev, act=ACT[act])
    ref, size = R.balance_grad(x64, i64, listed, act, d_loss)
    R.within(d.cpu(), ref, (2 * rel + 24 * R.U) * size + R.rounding(x.dtype, ref), "d_logits")


LARGE = [7e4, 1e8, 1.4e9, 2e9, 1e10, 2.5e10, 1e12, 1e20, 1e30, 9e37, 1.1e38, 3e38]


def far_logits(E, dtype, seed):
    """For each size, of either sign: one logit that large among ordinary ones, two that are alike, a whole row of it, a row of it
    and its lower neighbour, a row of it with one far lower; then rows of random sizes; every fourth row an ordinary one."""
    g = torch.Generator().manual_seed(seed)
    rows = []
    for size in LARGE:
        for v in (size, -size):
            one = torch.randn(E, generator=g).double()
            one[E // 2] = v
            two = torch.randn(E, generator=g).double()
            two[0] = two[E - 1] = v
            near = torch.full((E,), v, dtype=torch.float64).to(DTYPES[dtype])
            near[::2] = torch.nextafter(near, torch.full_like(near, -torch.inf))[::2]
            low = torch.full((E,), v, dtype=torch.float64)
            low[E // 3] = -3e38
            rows += [one, two, torch.full((E,), v, dtype=torch.float64), near.double(), low, torch.randn(E, generator=g).double()]
    for _ in range(60):
        top = 10.0 ** (4 + 34 * torch.rand((), generator=g).double()) * (1 if torch.rand((), generator=g) < 0.5 else -1)
        rows += [top + 3 * torch.randn(E, generator=g).double(), torch.where(torch.rand(E, generator=g) < 0.3, top, -top.abs()),
                 torch.randn(E, generator=g).double()]
    x = torch.stack(rows).to(DTYPES[dtype])
    assert torch.isfinite(x).all()
    return x.to(DEV)


@pytest.mark.parametrize("E,k", [(2, 1), (5, 2), (16, 4), (64, 6), (100, 8), (256, 8), (300, 16)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_selection_of_logits_far_from_0(E, k, dtype, act, renorm):
    check_topk(far_logits(E, dtype, E), k, act, renorm)


@pytest.mark.parametrize("E,k", [(2, 1), (5, 2), (16, 4), (64, 6), (100, 8), (256, 8), (300, 16)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("act", ["softmax", "sigmoid"])
def test_balance_of_logits_far_from_0(E, k, dtype, act):
    x = far_logits(E, dtype, E + 1)
    T = x.shape[0]
    check_balance(x, k, act, None)
    check_balance(x, k, act, [0, 1, 2, 7, 50, 51, T // 2, T - 3, T])


@pytest.mark.parametrize("T,E,act", [(6_000_000, 300, "softmax"), (6_000_000, 130, "sigmoid"), (12_000_000, 64, "softmax")])
def test_mean_probabilities_of_millions_of_rows(T, E, act):
    """Rows that are all alike: every addition of a probability rounds to the same side, and the error is that of the longest run of
    additions in fp32.  Runs of at most 64, and 8 to put them together, as in short batches."""
    row = torch.randn(E, generator=torch.Generator().manual_seed(E)).to(torch.bfloat16)
    x = row.to(DEV).repeat(T, 1)
    idx = torch.zeros((T, 1), dtype=torch.int32, device=DEV)
    loss, counts, mean_p, rows = mix.router_balance(x, idx, act=ACT[act])
    p = R.probabilities(row.double()[None], act)
    bound = row_bound(row[None], act) + 72 * R.U
    assert rows.item() == T and counts[0, 0].item() == T
    R.within(mean_p.cpu(), p, bound * p)
    R.within(loss.cpu(), E * p[:, 0], bound[0] * E * p[:, 0])


def ordinary_logits(T, E, dtype, seed, special=True):
    """Logits within some ten of each other, a few rows with experts forced in or out."""
    g = torch.Generator().manual_seed(seed)
    x = 2 * torch.randn((T, E), generator=g)
    if special and T >= 8:
        x[1] = -torch.inf
        x[2, E // 2:] = -torch.inf
        x[3, E // 3] = torch.inf
        x[5, 0] = torch.nan
        x[6] = torch.round(x[6])
    return x.to(DTYPES[dtype]).to(DEV)


@pytest.mark.parametrize("T,E,k", [(1, 8, 2), (64, 8, 2), (33, 9, 2), (40, 16, 16), (29, 31, 4), (70, 33, 6), (64, 64, 8), (31, 100, 16), (19, 160, 6), (50, 256, 8),
                                   (20, 257, 8), (24, 512, 16), (300, 64, 6)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("act,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_selection_with_a_bound_for_each_row(T, E, k, dtype, act, renorm):
    check_topk(ordinary_logits(T, E, dtype, T + E), k, act, renorm)


# more than 37888 rows in requests of fewer than 64: units of one warp and 32 rows; 62 rows in one segment and more than 16384 logits: units of
# one warp, their sums put together by a cluster; the others as they come
BALANCES = [(40000, 24, 3, "many"), (62, 300, 5, "one"), (63, 512, 8, "one"), (50000, 100, 6, "many"), (3000, 64, 6, "many"), (40, 8, 2, "one"),
            (517, 8, 2, "two"), (2500, 160, 8, "two"), (20000, 33, 4, "two")]


@pytest.mark.parametrize("T,E,k,kind", BALANCES)
@pytest.mark.parametrize("dtype,act", [("fp32", "softmax"), ("bf16", "softmax"), ("fp16", "sigmoid"), ("fp32", "sigmoid")])
def test_balance_with_a_bound_for_each_segment(T, E, k, kind, dtype, act):
    seg = None
    if kind == "two":
        seg = [0, T // 3, T - 5]
    elif kind == "many":                                       # ragged, some empty, the first and the last rows in none
        cuts = torch.randint(3, T - 9, (2000,), generator=torch.Generator().manual_seed(T)).tolist()
        seg = sorted(cuts + cuts[:200])
    check_balance(ordinary_logits(T, E, dtype, T + E), k, act, seg)
