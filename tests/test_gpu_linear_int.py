"""Products in 8-bit integers with a scale per token and output channel, alone and by experts, against 64 bits."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import operator_reference as R
import paper_2607_22595_b200 as mix

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(autouse=True)
def no_wait_ran_out():
    yield
    assert mix.linear_int_status() == 0


def _operands(T, K, N, seed, E=None):
    g = torch.Generator(device=DEV).manual_seed(seed)
    codes = torch.randint(-127, 128, (T, K), generator=g, device=DEV, dtype=torch.int8)
    W = torch.randint(-127, 128, (N, K) if E is None else (E, N, K), generator=g, device=DEV, dtype=torch.int8)
    scale = torch.rand(T, generator=g, device=DEV) * 0.02
    w_scale = torch.rand(W.shape[:-1], generator=g, device=DEV) * 0.01
    return codes, scale, W, w_scale


def _product(codes, scale, W, w_scale, bias=None):
    """float64: the product, and the bound of the fp32 arithmetic behind the exact sum (the sum as a float, two products)."""
    y = (codes.double() @ W.double().t()) * scale.double()[:, None] * w_scale.double()[None]
    bound = 3 * R.U * y.abs()
    if bias is not None:
        y = y + bias.double()[None]
        bound = bound + R.U * y.abs()
    return y, bound


@pytest.mark.parametrize("T,K,N", [(1, 16, 1), (1, 4096, 1000), (2, 32, 7), (15, 128, 128), (16, 144, 130), (17, 112, 300), (31, 1008, 129), (33, 256, 64),
                                   (64, 4096, 512), (65, 528, 1111), (127, 128, 2), (128, 640, 257), (129, 2048, 384), (200, 16, 640), (255, 272, 1000),
                                   (257, 1024, 255), (600, 1296, 777), (1030, 512, 2050), (3, 8192, 128), (300, 131056, 3), (16, 8192, 4096), (50, 2064, 1000),
                                   (100, 4096, 1500), (130, 4096, 3000), (333, 1024, 5000), (1000, 2048, 9000), (4200, 144, 300)])
@pytest.mark.parametrize("dtype,bias", [("bf16", False), ("fp16", True), ("fp32", True)])
def test_product(T, K, N, dtype, bias):
    codes, scale, W, w_scale = _operands(T, K, N, T + K + N)
    b = torch.randn(N, device=DEV) if bias else None
    out = mix.linear_int(codes, scale, W, w_scale, bias=b, dtype=DTYPES[dtype])
    ref, bound = _product(codes, scale, W, w_scale, b)
    R.within(out, ref, bound + R.rounding(out.dtype, ref))


def test_sums_are_exact_at_the_longest_row():
    K = 131056
    codes = torch.full((5, K), -128, dtype=torch.int8, device=DEV)
    codes[1] = 127
    codes[2, ::2] = 127
    W = torch.full((9, K), -128, dtype=torch.int8, device=DEV)
    W[3] = 127
    W[4, 1::2] = 127
    ones = torch.ones(9, device=DEV)
    out = mix.linear_int(codes, ones[:5], W, ones, dtype=torch.float32)
    assert torch.equal(out, (codes.double() @ W.double().t()).float())     # the exact sum, rounded once


def test_special_scales():
    codes, scale, W, w_scale = _operands(40, 64, 50, 1)
    scale[3], scale[4], scale[5] = 0.0, torch.nan, torch.inf
    codes[5] = torch.where(codes[5] == 0, 1, codes[5])
    out = mix.linear_int(codes, scale, W, w_scale, dtype=torch.float32)
    assert (out[3] == 0).all() and torch.isnan(out[4]).all() and not torch.isfinite(out[5]).any()
    assert torch.isfinite(out[[0, 1, 2] + list(range(6, 40))]).all()


@pytest.mark.parametrize("N,pad", [(96, 0), (96, 8), (96, 3), (95, 0), (95, 1), (260, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_rows_of_the_output_that_lie_apart(N, pad, dtype):
    T, K = 70, 160
    codes, scale, W, w_scale = _operands(T, K, N, 3)
    whole = torch.full((T + 2, N + pad), 5.0, dtype=DTYPES[dtype], device=DEV)
    out = whole[1:T + 1, :N]
    assert mix.linear_int(codes, scale, W, w_scale, out=out) is out
    ref, bound = _product(codes, scale, W, w_scale)
    R.within(out, ref, bound + R.rounding(out.dtype, ref))
    assert (whole[0] == 5).all() and (whole[T + 1] == 5).all() and (whole[:, N:] == 5).all()


def test_no_rows():
    codes, scale, W, w_scale = _operands(0, 64, 50, 1)
    assert mix.linear_int(codes, scale, W, w_scale).shape == (0, 50)
    codes, scale = mix.quantize_rows(torch.empty((0, 64), dtype=torch.bfloat16, device=DEV))
    assert codes.shape == (0, 64)
    none = torch.empty((0, 2), dtype=torch.int32, device=DEV)
    offsets, order, position = mix.expert_order(none, 4)
    y = mix.linear_int_grouped(codes, scale, torch.zeros((4, 8, 64), dtype=torch.int8, device=DEV), torch.zeros((4, 8), device=DEV), offsets)
    assert y.shape == (0, 8)
    assert mix.expert_combine(y, none.float(), position).shape == (0, 8)
    out = mix.expert_combine(y, torch.ones((3, 2), device=DEV), torch.zeros((3, 2), dtype=torch.int32, device=DEV))
    assert (out == 0).all()                                # a position that names no row does not count


def test_offsets_beyond_31_bits():
    T, K, N = 70000, 16, 32768
    codes, scale, W, w_scale = _operands(T, K, N, 5)
    out = mix.linear_int(codes, scale, W, w_scale)
    at = torch.tensor([0, 1, 255, 256, 65535, 65536, 65537, 69998, 69999], device=DEV)
    ref, bound = _product(codes[at], scale[at], W, w_scale)
    R.within(out[at], ref, bound + R.rounding(out.dtype, ref))
    position = torch.tensor([[69999], [-1], [65536]], dtype=torch.int32, device=DEV)
    back = mix.expert_combine(out, torch.ones((3, 1), device=DEV), position)
    assert torch.equal(back[0], out[69999]) and (back[1] == 0).all() and torch.equal(back[2], out[65536])


# ---------------------------------------------------------------------------------------------------- quantisation
@pytest.mark.parametrize("T,d", [(1, 16), (5, 48), (3, 1024), (4, 1040), (9, 4096), (2, 4112), (7, 5120), (2, 8192), (3, 8208), (2, 20000), (1, 131056)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_quantize_rows(T, d, dtype):
    g = torch.Generator(device=DEV).manual_seed(d)
    x = torch.randn((T, d), generator=g, device=DEV)
    x[0, ::3] *= 0.01
    x = x.to(DTYPES[dtype])
    if T > 2:
        x[1] = 0
        x[2] = torch.randint(-254, 255, (d,), generator=g, device=DEV).to(x.dtype)      # halves: a = 254 and whole numbers
        x[2, d // 2] = -254
    x[T - 1, 5] = x[T - 1].abs().max() * 2                 # x / a = 1 / 2, a half, where the first largest was
    codes, scale = mix.quantize_rows(x)
    ref, a = R.codes_of(x)
    assert torch.equal(codes.double(), ref)
    want = a.cpu().numpy().astype(np.float32) / np.float32(127)
    assert np.array_equal(scale.cpu().numpy(), want)


def test_quantize_rows_of_every_pair_of_values():
    """Every bf16 number against a set of largest values: each quotient, each half among them."""
    values = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).to(DEV)
    values = values[torch.isfinite(values) & (values >= 0)]
    for a in (1.0, 1.9921875, 254.0, 127.0, 3.0, 1e-38, 9.2e-41, 3.3e38, 0.0078125, 173.0):
        a = torch.tensor(a, device=DEV).to(torch.bfloat16)
        fit = values[values <= a]
        n = (fit.numel() + 16) // 16 * 16
        x = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
        x[:fit.numel()] = torch.where(torch.arange(fit.numel(), device=DEV) % 2 == 0, fit, -fit)
        x[-1] = a
        x = x[None]
        codes, scale = mix.quantize_rows(x)
        assert torch.equal(codes.double(), R.codes_of(x)[0]), a
        assert scale.item() == float(np.float32(a.item()) / np.float32(127))


def test_quantize_rows_of_every_pair_of_fp16_values():
    """The same for fp16, whose largest values that are multiples of 127 have halves everywhere."""
    values = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.float16).to(DEV)
    values = values[torch.isfinite(values) & (values >= 0)]
    for a in (1.0, 1.999, 127.0, 254.0, 1143.0, 1270.0, 1397.0, 1524.0, 1651.0, 1778.0, 1905.0, 2032.0, 381.0 / 64, 635.0 / 8, 1025.0, 2047.0, 65504.0, 6e-8,
              6.1e-5, 1143.0 * 2.0**-24, 173.0):
        a = torch.tensor(a, device=DEV).to(torch.float16)
        fit = values[values <= a]
        n = (fit.numel() + 16) // 16 * 16
        x = torch.zeros(n, dtype=torch.float16, device=DEV)
        x[:fit.numel()] = torch.where(torch.arange(fit.numel(), device=DEV) % 2 == 0, fit, -fit)
        x[-1] = a
        codes, scale = mix.quantize_rows(torch.stack([x, -x]))
        assert torch.equal(codes.double(), R.codes_of(torch.stack([x, -x]))[0]), a
        assert scale[0].item() == float(np.float32(a.item()) / np.float32(127))


def test_quantize_rows_with_infinities_and_nan():
    x = torch.randn((6, 96), device=DEV).to(torch.bfloat16)
    x[1, 7], x[2, 95], x[3, 0], x[4, 3] = torch.inf, -torch.inf, torch.nan, torch.nan
    x[4, 4] = 1e30
    codes, scale = mix.quantize_rows(x)
    assert torch.isnan(scale[1:5]).all() and (codes[1:5] == 0).all() and torch.isfinite(scale[[0, 5]]).all()
    W, w_scale = torch.randint(-5, 5, (33, 96), device=DEV, dtype=torch.int8), torch.ones(33, device=DEV)
    y = mix.linear_int(codes, scale, W, w_scale)
    assert torch.isnan(y[1:5]).all() and torch.isfinite(y[[0, 5]]).all()


@pytest.mark.parametrize("d,pad,shift", [(64, 0, 1), (64, 8, 0), (64, 5, 3), (5120, 8, 8), (5120, 1, 0), (1056, 24, 1)])
def test_quantize_rows_that_lie_apart(d, pad, shift):
    T = 11
    base = torch.full((T * (d + pad) + shift,), torch.nan, dtype=torch.bfloat16, device=DEV)
    x = base[shift:].view(T, d + pad)[:, :d]
    x.copy_(torch.randn((T, d), device=DEV))
    codes, scale = mix.quantize_rows(x)
    assert torch.equal(codes.double(), R.codes_of(x)[0])
    order = torch.tensor([21, 0, -1, 5, 5, 22, 19, -7, 2**31 - 1], dtype=torch.int32, device=DEV)        # 22 // 2 names no row
    got, got_scale = mix.quantize_rows(x, order=order, k=2)
    for i, t in enumerate([10, 0, None, 2, 2, None, 9, None, None]):
        assert torch.equal(got[i], codes[t] if t is not None else torch.zeros_like(codes[0]))
        assert got_scale[i] == (scale[t] if t is not None else 0)


# ---------------------------------------------------------------------------------------------------- by experts
def _counts(kind, E, seed):
    g = torch.Generator().manual_seed(seed)
    c = {"even": torch.full((E,), 5), "one": torch.zeros(E, dtype=torch.long), "few": torch.randint(0, 3, (E,), generator=g),
         "ragged": torch.randint(0, 70, (E,), generator=g), "large": torch.randint(0, 600, (E,), generator=g)}[kind]
    if kind == "one":
        c[E // 2] = 300
    return c.tolist()


@pytest.mark.parametrize("E,kind", [(1, "even"), (2, "one"), (3, "large"), (8, "even"), (8, "few"), (8, "ragged"), (5, "large"), (33, "ragged"), (64, "few"),
                                    (100, "one"), (512, "few")])
@pytest.mark.parametrize("K,N,dtype,bias", [(64, 48, "bf16", False), (208, 129, "fp16", True), (512, 384, "fp32", False), (4112, 160, "bf16", True)])
def test_grouped_product(E, kind, K, N, dtype, bias):
    counts = _counts(kind, E, E)
    front, tail = (3, 7) if E % 2 else (0, 0)
    n = sum(counts) + front + tail
    codes, scale, W, w_scale = _operands(n, K, N, E + K, E=E)
    b = torch.randn((E, N), device=DEV) if bias else None
    offsets = torch.tensor([front + sum(counts[:i]) for i in range(E + 1)], dtype=torch.int32, device=DEV)
    out = torch.full((n, N), 3.0, dtype=DTYPES[dtype], device=DEV)
    mix.linear_int_grouped(codes, scale, W, w_scale, offsets, bias=b, out=out)
    at = offsets.tolist()
    for e in range(E):
        rows = slice(at[e], at[e + 1])
        ref, bound = _product(codes[rows], scale[rows], W[e], w_scale[e], None if b is None else b[e])
        R.within(out[rows], ref, bound + R.rounding(out.dtype, ref), "expert %d" % e)
    assert (out[:front] == 3).all() and (out[at[E]:] == 3).all()


def test_offsets_that_leave_the_rows_or_fall_are_held_in():
    codes, scale, W, w_scale = _operands(50, 64, 40, 2, E=4)
    good = torch.tensor([0, 20, 20, 50, 50], dtype=torch.int32, device=DEV)
    bad = torch.tensor([-9, 20, 11, 2**31 - 1, 7], dtype=torch.int32, device=DEV)
    assert torch.equal(mix.linear_int_grouped(codes, scale, W, w_scale, good), mix.linear_int_grouped(codes, scale, W, w_scale, bad))


@pytest.mark.parametrize("T,k,N,dtype", [(1, 1, 1, "bf16"), (5, 2, 8, "fp32"), (7, 3, 100, "fp16"), (40, 8, 4096, "bf16"), (3, 16, 5000, "fp32"), (9, 2, 8200, "bf16"),
                                         (700, 6, 64, "bf16")])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_combine(T, k, N, dtype, pad):
    g = torch.Generator(device=DEV).manual_seed(T + N)
    n = T * k
    y = torch.randn((n, N + pad), generator=g, device=DEV).to(DTYPES[dtype])[:, :N]
    w = torch.randn((T, k), generator=g, device=DEV)
    position = torch.randperm(n, generator=g, device=DEV).int().view(T, k)
    if n > 4:
        position[0] = -1                                   # a token without experts
        position[1, 0] = n                                 # names no row
        position[2, 0] = position[2, k - 1]                # the same row twice
        w[0] = torch.nan
    out = torch.full((T, N + pad), 9.0, dtype=y.dtype, device=DEV)
    mix.expert_combine(y, w, position, out=out[:, :N])
    there = (position >= 0) & (position < n)
    terms = torch.where(there, w, 0.0).double()[:, :, None] * y[position.clamp(0, n - 1).long()].double()
    R.within(out[:, :N], terms.sum(1), k * R.U * terms.abs().sum(1) + R.rounding(y.dtype, terms.sum(1)))
    assert (out[:, N:] == 9).all()


# ---------------------------------------------------------------------------------------------------- together
def _layer(m, logits, hidden, W, w_scale, k, n_live, seg):
    m.apply_router(logits)
    idx, weights = mix.router_topk(logits, k, n_live=n_live)
    offsets, order, position = mix.expert_order(idx, W.shape[0])
    codes, scale = mix.quantize_rows(hidden, order=order, k=k)
    y = mix.linear_int_grouped(codes, scale, W, w_scale, offsets, dtype=hidden.dtype)
    return (mix.expert_combine(y, weights, position), idx, *mix.router_balance(logits, idx, seg))


@pytest.mark.parametrize("T,E,k,K,N", [(1, 8, 2, 64, 64), (24, 8, 2, 128, 200), (150, 40, 6, 320, 136)])
def test_a_steered_moe_layer_eager_and_replayed(T, E, k, K, N):
    """Router steering by the hook, then selection, order, the experts' products, their sum and the requests' loads."""
    g = torch.Generator(device=DEV).manual_seed(T)
    m = mix.Mix(d_model=64, T_max=T, n_slots_max=2)
    delta = torch.zeros(E, device=DEV)
    delta[1], delta[2] = -torch.inf, torch.inf             # expert 1 out, expert 2 in
    m.register_router(0, delta)
    slots = torch.where(torch.arange(T) % 3 == 0, 0, -1).int().to(DEV)
    live = max(1, T - T // 5)
    n_live = torch.tensor([live], dtype=torch.int32, device=DEV)
    seg = torch.tensor([0, live // 2, live], dtype=torch.int32, device=DEV)
    W32 = torch.randn((E, N, K), generator=g, device=DEV).to(torch.bfloat16)
    W, w_scale = mix.quantize_rows(W32.view(E * N, K))
    W, w_scale = W.view(E, N, K), w_scale.view(E, N)
    logits, hidden = torch.empty((T, E), device=DEV), torch.empty((T, K), dtype=torch.bfloat16, device=DEV)

    def check(out, raw):
        x = raw.clone()
        x[slots == 0] += delta
        ref_idx, ref_w = R.topk(x, k, "softmax", True, live)
        assert torch.equal(out[1].cpu().long(), ref_idx)
        if live > 3:
            assert (ref_idx[3] == 2).any() and not (ref_idx[3] == 1).any()
        codes, a = R.codes_of(hidden)
        ref = torch.zeros((T, N), dtype=torch.float64, device=DEV)
        size = torch.zeros_like(ref)
        for t in range(live):
            for j in range(k):
                e = int(ref_idx[t, j])
                if e < 0:
                    continue
                y = (codes[t] @ W[e].double().t()) * (a[t] / 127) * w_scale[e].double()
                ref[t] += ref_w[t, j].item() * y
                size[t] += ref_w[t, j].item() * y.abs()
        # per term: the row's scale (U), the product's three roundings, y's half step, the weight, the sum's k additions
        bound = (R.half_step(hidden.dtype) + (5 + k) * R.U + R.rel_p(raw, "softmax")) * size * (1 + R.half_step(hidden.dtype))
        R.within(out[0], ref, bound + R.rounding(hidden.dtype, ref))
        r_loss, r_counts, _, r_rows = R.balance(x.cpu().double(), ref_idx, seg.tolist(), "softmax")
        assert torch.equal(out[3].cpu().long(), r_counts) and out[5].tolist() == r_rows
        R.within(out[2].cpu(), r_loss, (R.rel_p(raw, "softmax") + 72 * R.U) * r_loss + 1e-37)

    def fill(seed):
        gg = torch.Generator(device=DEV).manual_seed(seed)
        raw = 2 * torch.randn((T, E), generator=gg, device=DEV)
        logits.copy_(raw)
        hidden.copy_(torch.randn((T, K), generator=gg, device=DEV))
        return raw

    m.set_slot_map(slots)
    raw = fill(1)
    check(_layer(m, logits, hidden, W, w_scale, k, n_live, seg), raw)
    raw = fill(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _layer(m, logits, hidden, W, w_scale, k, n_live, seg)
    for seed in (2, 3):
        raw = fill(seed)
        graph.replay()
        check(out, raw)
    m.destroy()


def test_two_graphs_and_two_streams_at_once():
    """Calls on two streams, eager and replayed, share no scratch memory."""
    def make(seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        T, E, k, K, N = 3000, 32, 4, 256, 256
        logits = torch.randn((T, E), generator=g, device=DEV)
        hidden = torch.randn((T, K), generator=g, device=DEV).to(torch.bfloat16)
        W = torch.randint(-127, 128, (E, N, K), generator=g, device=DEV, dtype=torch.int8)
        ws = torch.rand((E, N), generator=g, device=DEV)

        def step():
            idx, w = mix.router_topk(logits, k)
            offsets, order, position = mix.expert_order(idx, E)
            codes, scale = mix.quantize_rows(hidden, order=order, k=k)
            y = mix.linear_int_grouped(codes, scale, W, ws, offsets)
            return (mix.expert_combine(y, w, position), *mix.router_balance(logits, idx))
        return step

    steps = [make(1), make(2)]
    want = [[t.clone() for t in s()] for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs, outs = [], []
    for s in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(s())
        graphs.append(graph)
    for _ in range(5):
        eager = []
        for s, stream, graph in zip(steps, streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
                eager.append(s())
        torch.cuda.synchronize()
        for w, a, b in zip(want, outs, eager):
            assert all(torch.equal(x, y) for x, y in zip(w, a)) and all(torch.equal(x, y) for x, y in zip(w, b))


def test_a_stream_given_by_argument():
    x = torch.randn((500, 128), device=DEV).to(torch.bfloat16)
    idx = torch.randint(0, 16, (3000, 2), device=DEV, dtype=torch.int32)
    want = mix.expert_order(idx, 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = mix.expert_order(idx, 16, stream=side)
    codes, scale = mix.quantize_rows(x, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(codes.double(), R.codes_of(x)[0])


def test_the_first_calls_of_a_process_may_be_captured():
    """Nothing has to be called before a capture, nor in a warm-up."""
    code = """
import torch, paper_2607_22595_b200 as mix
g = torch.Generator(device="cuda").manual_seed(1)
logits = torch.randn((40, 8), generator=g, device="cuda")
x = torch.randn((40, 64), generator=g, device="cuda").to(torch.bfloat16)
W = torch.randint(-9, 9, (8, 48, 64), generator=g, device="cuda", dtype=torch.int8)
ws = torch.ones((8, 48), device="cuda")
def step():
    idx, w = mix.router_topk(logits, 2)
    offsets, order, position = mix.expert_order(idx, 8)
    codes, scale = mix.quantize_rows(x, order=order, k=2)
    y = mix.linear_int_grouped(codes, scale, W, ws, offsets)
    loss, counts, mean_p, rows = mix.router_balance(logits, idx)
    return mix.expert_combine(y, w, position), mix.linear_int(codes, scale, W[0], ws[0]), mix.router_balance_grad(logits, idx, counts, rows, loss)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = step()
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(out, step()))
assert mix.linear_int_status() == 0
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr[-2000:]


def test_refused_tensors():
    codes, scale, W, w_scale = _operands(20, 64, 30, 1)
    grouped = _operands(20, 64, 30, 1, E=2)
    offsets = torch.tensor([0, 5, 20], dtype=torch.int32, device=DEV)
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    position = torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    for call in (lambda: mix.linear_int(codes.float(), scale, W, w_scale), lambda: mix.linear_int(codes, scale[:19], W, w_scale),
                 lambda: mix.linear_int(codes, scale, W[:, :48], w_scale), lambda: mix.linear_int(codes, scale, W, w_scale.double()),
                 lambda: mix.linear_int(codes, scale, W, w_scale, bias=w_scale[:5]), lambda: mix.linear_int(codes, scale, W, w_scale, dtype=torch.float64),
                 lambda: mix.linear_int(codes, scale, W, w_scale, out=torch.empty((20, 31), device=DEV)), lambda: mix.linear_int(codes, scale, W, w_scale, dtype=3),
                 lambda: mix.linear_int(codes, scale, grouped[2], grouped[3]), lambda: mix.linear_int_grouped(codes, scale, W, w_scale, offsets),
                 lambda: mix.linear_int_grouped(codes, scale, grouped[2], grouped[3], None),
                 lambda: mix.linear_int_grouped(codes, scale, grouped[2], grouped[3], offsets[:2]),
                 lambda: mix.linear_int_grouped(codes, scale, grouped[2], grouped[3], offsets.long()),
                 lambda: mix.quantize_rows(x, order=offsets.long()), lambda: mix.quantize_rows(x, order=offsets, k=0),
                 lambda: mix.quantize_rows(x, codes=torch.empty((4, 64), device=DEV)), lambda: mix.expert_combine(x, torch.zeros((4, 3), device=DEV), position),
                 lambda: mix.expert_combine(x, torch.zeros((4, 2), device=DEV), position, out=torch.empty((4, 64), device=DEV))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: mix.quantize_rows(x.float()), lambda: mix.quantize_rows(x[:, :40].contiguous()),
                 lambda: mix.linear_int(codes[:, :40].contiguous(), scale, W[:, :40].contiguous(), w_scale)):
        with pytest.raises(mix.MixError):
            call()


@pytest.mark.parametrize("T,k,N,dtype", [(1, 1, 1, "bf16"), (5, 2, 8, "fp32"), (7, 3, 100, "fp16"), (40, 8, 4096, "bf16"), (3, 16, 5000, "fp32"), (9, 2, 8200, "bf16"),
                                         (700, 6, 64, "bf16"), (0, 2, 16, "fp32")])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_gradients_of_combine(T, k, N, dtype, pad):
    g = torch.Generator(device=DEV).manual_seed(T + N)
    n = T * k + 3
    y = torch.randn((n, N + pad), generator=g, device=DEV).to(DTYPES[dtype])[:, :N]
    d_out = torch.randn((T, N + pad), generator=g, device=DEV).to(DTYPES[dtype])[:, :N]
    w = torch.randn((T, k), generator=g, device=DEV)
    position = torch.randperm(n, generator=g, device=DEV)[:T * k].int().view(T, k)
    if T > 4:
        position[0] = -1
        position[1, 0] = n
        w[0] = torch.nan
    d_y = torch.full((n, N + pad), 6.0, dtype=y.dtype, device=DEV)
    d_w, got = mix.expert_combine_grad(d_out, y, w, position, want_y=True, d_y=d_y[:, :N])
    assert torch.equal(mix.expert_combine_grad(d_out, y, w, position), d_w)
    there = (position >= 0) & (position < n)
    at = position.clamp(0, n - 1).long()
    terms = torch.where(there[:, :, None], d_out.double()[:, None] * y[at].double(), 0.0)
    # a thread's share one after the other (N / 256 additions, vectors of 8 within), a tree of 8 steps over the block
    R.within(d_w, terms.sum(2), (N / 256 + 8 + 16) * R.U * terms.abs().sum(2) + 1e-37, "d_weights")
    want = torch.full((n, N), 6.0, dtype=torch.float64, device=DEV)
    want[at[there]] = (w[:, :, None].double() * d_out.double()[:, None])[there]
    R.within(d_y[:, :N], want, R.U * want.abs() + R.rounding(y.dtype, want), "d_y")
    assert (d_y[:, N:] == 6).all() and torch.equal(got, d_y[:, :N])


def test_the_gradient_of_a_steering_against_differences():
    """A loss on the layer's output and its balance, through the sum over experts, the selection and the steering: all in one step, captured
    and replayed, against differences of the same in 64 bits (the chosen experts and their results held)."""
    T, E, k, K, N = 48, 12, 3, 64, 40
    g = torch.Generator(device=DEV).manual_seed(3)
    base = 1.5 * torch.randn((T, E), generator=g, device=DEV)
    delta = 0.3 * torch.randn(E, generator=g, device=DEV)
    hidden = torch.randn((T, K), generator=g, device=DEV).to(torch.bfloat16)
    W, w_scale = mix.quantize_rows((torch.randn((E * N, K), generator=g, device=DEV) / 8).to(torch.bfloat16))
    W, w_scale = W.view(E, N, K), w_scale.view(E, N)
    d_out = torch.randn((T, N), generator=g, device=DEV)
    seg = torch.tensor([0, 20, T], dtype=torch.int32, device=DEV)
    d_loss = torch.tensor([0.7, -0.4], device=DEV)
    m = mix.Mix(d_model=64, T_max=T, n_slots_max=1)
    m.register_router(0, delta)
    m.set_slot_map(torch.zeros(T, dtype=torch.int32, device=DEV))
    logits = torch.empty_like(base)

    def step():
        logits.copy_(base)
        m.apply_router(logits)
        idx, w = mix.router_topk(logits, k)
        offsets, order, position = mix.expert_order(idx, E)
        codes, scale = mix.quantize_rows(hidden, order=order, k=k)
        y = mix.linear_int_grouped(codes, scale, W, w_scale, offsets, dtype=torch.float32)
        d_w = mix.expert_combine_grad(d_out, y, w, position)
        loss, counts, _, rows = mix.router_balance(logits, idx, seg)
        d = mix.router_topk_grad(logits, idx, w, d_w)
        b = mix.router_balance_grad(logits, idx, counts, rows, d_loss, seg)
        return idx, position, y, d, b

    eager = [t.clone() for t in step()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(eager, out))
    idx, position, y, d, b = (t.cpu() for t in eager)
    y64, i64, p = y.double(), idx.long(), position.long()
    base64, G, seg64 = base.cpu().double(), d_out.cpu().double(), seg.tolist()
    dl = d_loss.cpu().double()

    def f(x):
        w = R.weights_of(x, i64, "softmax", True)
        return ((w[:, :, None] * y64[p]).sum(1) * G).sum() + (R.balance(x, i64, seg64, "softmax")[0] * dl).sum()

    # base + delta is rounded to fp32 by the steering: the differences are taken around what it gave
    x = (base.cpu() + delta.cpu()).double()
    assert torch.equal(logits.cpu().double(), x)
    d_delta = (d.double() + b.double()).sum(0)
    # the kernel's own error: of the weights' gradients (their dot products and the selection's bound), of the balance's
    d_w = (G[:, None] * y64[p]).sum(2)
    size_w = (G[:, None] * y64[p]).abs().sum(2)
    _, size = R.topk_grad(x, i64, "softmax", True, size_w)
    _, bsize = R.balance_grad(x, i64, seg64, "softmax", dl)
    own = ((2 * R.rel_p(x, "softmax") + 60 * R.U) * (size + bsize)).sum(0)
    h = 1e-5
    for e in range(E):
        up = x.clone(); up[:, e] += h
        down = x.clone(); down[:, e] -= h
        change = (f(up) - f(down)) / (2 * h)
        # of the differences: 2^-53 |f| / h and h^2 / 6 times third derivatives of at most 6 sum |d_w| (and 6 E)
        assert abs(change - d_delta[e]) <= own[e] + 1e-10 * (6 * d_w.abs().sum() + 6 * E) + 1e-9, e
    m.destroy()
