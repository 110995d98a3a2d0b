"""The bounded waits of the 8-bit products run out: failure detection without a GPU fault."""
import pytest
import torch

import operator_reference as R
import paper_2607_22595_b200 as mix

pytestmark = pytest.mark.gpu
DEV = "cuda"
WAIT_TIMEOUT = 4


def _operands(T, K, N, E=None):
    g = torch.Generator(device=DEV).manual_seed(T + K + N)
    codes = torch.randint(-127, 128, (T, K), generator=g, device=DEV, dtype=torch.int8)
    W = torch.randint(-127, 128, (N, K) if E is None else (E, N, K), generator=g, device=DEV, dtype=torch.int8)
    return codes, torch.rand(T, generator=g, device=DEV), W, torch.rand(W.shape[:-1], generator=g, device=DEV)


# tiles of single CTAs (32, 64 and 128 tokens), CTA pairs, and clusters of 2, 4 and 8 CTAs that share a tile's codes
@pytest.mark.parametrize("T,K,N,E", [(20, 256, 300, None), (20, 256, 20000, None), (60, 512, 9000, None), (100, 512, 20000, None), (4200, 512, 700, None),
                                     (16, 1024, 4096, None), (16, 4096, 4096, None), (16, 14336, 128, None), (600, 512, 256, 5), (30, 512, 256, 4)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_waits_that_run_out_raise_the_status_and_leave_the_rest_usable(T, K, N, E, dtype):
    codes, scale, W, w_scale = _operands(T, K, N, E)
    whole = torch.full((T + 2, N + 5), 3.0, dtype=dtype, device=DEV)
    out = whole[1:T + 1, :N]
    offsets = None if E is None else torch.tensor([T * i // E for i in range(E + 1)], dtype=torch.int32, device=DEV)

    def call():
        if E is None:
            mix.linear_int(codes, scale, W, w_scale, out=out)
        else:
            mix.linear_int_grouped(codes, scale, W, w_scale, offsets, out=out)

    lib = mix.load_library()
    assert mix.linear_int_status() == 0
    assert lib.mix_debug_linear_int_stall(1) == 0
    try:
        call()
        call()
    finally:
        assert lib.mix_debug_linear_int_stall(0) == 1
    assert mix.linear_int_status() == WAIT_TIMEOUT         # returns: nothing hangs
    assert mix.linear_int_status() == 0                    # reading the word clears it
    assert (whole[0] == 3).all() and (whole[-1] == 3).all() and (whole[:, N:] == 3).all()
    call()                                                 # and the next call on the same device is right
    for e in range(E or 1):
        rows, w, ws = (slice(None), W, w_scale) if E is None else (slice(T * e // E, T * (e + 1) // E), W[e], w_scale[e])
        ref = (codes[rows].double() @ w.double().t()) * scale[rows].double()[:, None] * ws.double()[None]
        R.within(out[rows], ref, 3 * R.U * ref.abs() + R.rounding(dtype, ref))
    assert mix.linear_int_status() == 0


def test_the_status_call_is_refused_in_a_capture_that_goes_on():
    codes, scale, W, w_scale = _operands(20, 64, 64)
    want = mix.linear_int(codes, scale, W, w_scale)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(mix.MixError) as e:
            mix.linear_int_status()
        out = mix.linear_int(codes, scale, W, w_scale)
    assert e.value.code == -3
    graph.replay()
    assert torch.equal(out, want) and mix.linear_int_status() == 0


def test_a_wait_that_runs_out_while_the_status_is_read_is_not_lost():
    """A product of one CTA runs into its time-out on one stream while another reads the word over and over."""
    codes, scale, W, w_scale = _operands(20, 64, 64)
    lib = mix.load_library()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    assert mix.linear_int_status() == 0
    for trial in range(400):
        lib.mix_debug_linear_int_stall(1)
        try:
            mix.linear_int(codes, scale, W, w_scale, stream=side)
        finally:
            lib.mix_debug_linear_int_stall(0)
        seen = 0
        while not side.query():
            seen |= mix.linear_int_status()
        assert seen | mix.linear_int_status() == WAIT_TIMEOUT, trial
