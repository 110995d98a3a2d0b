"""Calls behind the router on a stream given by argument, beside work on the current one."""
import pytest
import torch

import paper_2607_22595_b200 as mix

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _inputs(seed, T=6000, k=4, E=40):
    g = torch.Generator(device=DEV).manual_seed(seed)
    idx = torch.randint(0, E, (T, k), generator=g, device=DEV, dtype=torch.int32)
    return idx, torch.randn((T, E), generator=g, device=DEV), E


def _streams_with_memory():
    return {segment["stream"] for segment in torch.cuda.memory_snapshot()}


@pytest.mark.parametrize("as_number", [False, True])
def test_outputs_and_scratch_are_allocated_on_the_given_stream(as_number):
    idx, logits, E = _inputs(1)
    T, k = idx.shape
    given = [torch.empty(n, dtype=torch.int32, device=DEV) for n in (E + 1, T * k)] + [torch.empty((T, k), dtype=torch.int32, device=DEV)]
    torch.cuda.synchronize()
    before = torch.cuda.current_stream()
    for call in (lambda s: mix.expert_order(idx, E, *given, stream=s), lambda s: mix.router_balance(logits, idx, stream=s),
                 lambda s: mix.router_topk(logits, k, stream=s), lambda s: mix.quantize_rows(logits[:, :32].bfloat16(), stream=s)):
        torch.cuda.empty_cache()
        used = _streams_with_memory()
        side = next(s for s in (torch.cuda.Stream() for _ in range(64)) if s.cuda_stream not in used)    # (torch hands out 32 in turn)
        torch.cuda.synchronize()
        out = call(side.cuda_stream if as_number else side)
        assert side.cuda_stream in _streams_with_memory()
        assert torch.cuda.current_stream() == before
        side.synchronize()
        del out


def test_the_current_stream_and_a_given_one_share_no_scratch():
    """Calls with scratch memory, in turn on the current stream and on another, nothing waiting in between."""
    sets = [_inputs(2), _inputs(3)]
    want = [[t.clone() for t in (*mix.expert_order(i, E), *mix.router_balance(x, i))] for i, x, E in sets]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = []
    for _ in range(30):
        for (i, x, E), stream in zip(sets, (None, side)):
            out.append((*mix.expert_order(i, E, stream=stream), *mix.router_balance(x, i, stream=stream)))
    torch.cuda.synchronize()
    for n, got in enumerate(out):
        assert all(torch.equal(a, b) for a, b in zip(got, want[n % 2]))


def test_results_dropped_while_the_current_stream_reads_them():
    """A result of a given stream that is read on the current one and dropped at once is not handed out before the read is over."""
    idx, logits, E = _inputs(4)
    want = mix.router_balance(logits, idx)[2].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    reads = []
    for _ in range(5):
        mean = mix.router_balance(logits, idx, stream=side)[2]
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda._sleep(2000000)
        reads.append(mean.clone())
        del mean
        with torch.cuda.stream(side):
            torch.full((4 * E + 2048,), 7.0, device=DEV)   # the size class of the call's outputs
    torch.cuda.synchronize()
    assert all(torch.equal(r, want) for r in reads)


def test_a_given_stream_inside_a_capture():
    idx, logits, E = _inputs(5)
    want = [t.clone() for t in (*mix.expert_order(idx, E), *mix.router_balance(logits, idx))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        one = mix.expert_order(idx, E, stream=side)
        two = mix.router_balance(logits, idx)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*one, *two), want))
