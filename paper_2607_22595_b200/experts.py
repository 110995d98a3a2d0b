"""Behind the router: selection, balance and the experts' products in 8-bit integers.

    m.apply_router(logits)                                          # steer (a Mix context), then, without a context:
    idx, weights = mix.router_topk(logits, k)                       # the experts of each token
    offsets, order, position = mix.expert_order(idx, n_experts)     # the tokens by expert
    codes, scale = mix.quantize_rows(hidden, order=order, k=k)      # 8-bit rows, each expert's next to each other
    y = mix.linear_int_grouped(codes, scale, W, w_scale, offsets)   # each expert's product
    out = mix.expert_combine(y, weights, position)                  # summed over each token's experts
    loss, counts, mean_p, rows = mix.router_balance(logits, idx, seg)   # what the steering did to each request's load

Every function works on the device of its tensors, on the stream given or that device's current one.  Outputs that are not given, and
scratch memory, are allocated by torch on that stream (outputs of one call share one allocation); inputs and outputs that are given must be
ready there, and whoever reads the results on another stream waits for that one first.  Gradients
are functions of their own: nothing here records a graph.
A tensor of the wrong type, shape or place raises ValueError, what the library refuses MixError.
The C ABI (include/mix.h) states the arithmetic; the checks and the calls into it are in csrc/fastops.cpp.
"""
from __future__ import annotations

import ctypes as C
import re

import torch

from . import binding as B
from .binding import MIX_ACT_SIGMOID, MIX_ACT_SOFTMAX, MixError  # noqa: F401


_loaded = None        # the module of these calls (csrc/fastops.cpp)


def _ops():
    """Loaded by the first of these calls: it is linked to torch's C++ libraries, which the hook does without."""
    global _loaded
    if _loaded is None:
        B.load_library()
        here = re.match(r"[0-9.]*", torch.__version__).group().rstrip(".")   # (of 2.11.0a0+git as well)
        try:
            from . import _fastops
        except ImportError as e:
            raise RuntimeError("_fastops.so does not load with torch %s: run __graft_entry__.build() again (%s)" % (here, e)) from e
        if _fastops.torch_version != here:
            raise RuntimeError("_fastops.so was built for torch %s, not %s: run __graft_entry__.build() again" % (_fastops.torch_version, here))
        _loaded = _fastops
    return _loaded


def router_topk(logits, k, act=MIX_ACT_SOFTMAX, renormalise=True, n_live=None, idx=None, weights=None, stream=None):
    """The k largest logits of each row -> idx int32 [T, k] (largest first, of equal ones the lower index first) and weights
    fp32 [T, k]: their softmax or sigmoid values, divided by their sum where `renormalise`.  logits: fp32, bf16 or fp16
    [T, n_experts].  -inf and NaN are never chosen (-1, weight 0, where fewer than k are left), +inf shares the row.  n_live: int32[1]
    on the device; rows from there on are padding and get -1 and 0.  New outputs are parts of one allocation: who keeps or saves the one
    keeps or saves both (clone it, or give buffers)."""
    return (_loaded or _ops()).router_topk(logits, k, act, renormalise, n_live, idx, weights, stream)


def router_topk_grad(logits, idx, weights, d_weights, act=MIX_ACT_SOFTMAX, renormalise=True, d_logits=None, stream=None):
    """Gradient of router_topk's weights with respect to the logits: d_logits [T, n_experts] in the logits' type."""
    return (_loaded or _ops()).router_topk_grad(logits, idx, weights, d_weights, act, renormalise, d_logits, stream)


def expert_order(idx, n_experts, offsets=None, order=None, position=None, stream=None):
    """The entries of idx int32 [T, k] sorted by expert, stably -> offsets int32 [n_experts + 1], order int32 [T * k] (entries
    t * k + j, -1 behind the last), position int32 [T, k] (the entry's place in `order`, -1 where it names no expert).  New outputs are
    parts of one allocation."""
    return (_loaded or _ops()).expert_order(idx, n_experts, offsets, order, position, stream)


def router_balance(logits, idx, seg=None, act=MIX_ACT_SOFTMAX, stream=None):
    """Per segment of rows (seg int32 [n + 1], offsets on the device; None: all rows are one segment): the balance loss fp32 [n], how
    often each expert was chosen int32 [n, n_experts], the experts' mean probabilities fp32 [n, n_experts] and the rows counted
    int32 [n].  idx int32 [T, k] as from router_topk; rows that name no expert do not count.  The four are parts of one allocation: who keeps
    the loss keeps counts and mean probabilities too (clone it)."""
    return (_loaded or _ops()).router_balance(logits, idx, seg, act, stream)


def router_balance_grad(logits, idx, counts, rows, d_loss, seg=None, act=MIX_ACT_SOFTMAX, d_logits=None, stream=None):
    """Gradient of router_balance's losses with respect to the logits, for d_loss fp32 [n] and the counts and rows that it gave."""
    return (_loaded or _ops()).router_balance_grad(logits, idx, counts, rows, d_loss, seg, act, d_logits, stream)


def quantize_rows(x, order=None, k=1, codes=None, scale=None, stream=None):
    """Rows of x (bf16 or fp16 [T, d], d a multiple of 16) as 8-bit integers: codes int8 [n, d] and scale fp32 [n], codes * scale being
    the nearest to x.  With `order` (expert_order's, int32 [n]) row i is row order[i] // k of x; entries of -1 give zeros.  New outputs are parts of one allocation."""
    return (_loaded or _ops()).quantize_rows(x, order, k, codes, scale, stream)


def linear_int(codes, scale, W, w_scale, bias=None, out=None, dtype=torch.bfloat16, stream=None):
    """out[t, n] = (codes[t] . W[n]) scale[t] w_scale[n] + bias[n], the product of 8-bit integers exact, in `dtype` (or out's type).
    codes int8 [T, K], scale fp32 [T]; W int8 [N, K], w_scale fp32 [N], bias fp32 [N]."""
    return (_loaded or _ops()).linear_int(codes, scale, W, w_scale, None, bias, out, dtype, stream)


def linear_int_grouped(codes, scale, W, w_scale, offsets, bias=None, out=None, dtype=torch.bfloat16, stream=None):
    """linear_int with a weight set per group of rows: rows offsets[e] .. offsets[e + 1) of codes (int8 [n, K]) go through W[e]
    (int8 [n_experts, N, K]; w_scale and bias fp32 [n_experts, N]).  Rows of `out` that belong to no expert are left as they were."""
    if offsets is None:
        raise ValueError("offsets must be a CUDA tensor")
    return (_loaded or _ops()).linear_int(codes, scale, W, w_scale, offsets, bias, out, dtype, stream)


def linear_int_status(stream=None) -> int:
    """The status bits of the 8-bit products on the current device since the last call (MIX_STATUS_WAIT_TIMEOUT or 0); synchronises."""
    bits, err = C.c_uint(0), C.create_string_buffer(256)
    rc = B.load_library().mix_linear_int_status(C.byref(bits), B._stream(stream), err, 256)
    if rc != 0:
        raise MixError(rc, err.value.decode())
    return int(bits.value)


def expert_combine(y, weights, position, out=None, stream=None):
    """out[t] = sum_j weights[t, j] y[position[t, j]] -> [T, N] in y's type.  y [n, N] in expert_order's order; entries of -1 do not count.
    The sum is taken in fp32; results in 16 bits have been rounded before it, fp32 ones (linear_int_grouped's dtype) have not."""
    return (_loaded or _ops()).expert_combine(y, weights, position, out, stream)


def expert_combine_grad(d_out, y, weights, position, want_y=False, d_weights=None, d_y=None, stream=None):
    """Gradients of expert_combine for d_out [T, N]: d_weights fp32 [T, k] -- router_topk_grad takes it from there -- and with want_y
    also d_y [n, N], of which rows that no entry of `position` names are left as they were (uninitialised if d_y is not given)."""
    return (_loaded or _ops()).expert_combine_grad(d_out, y, weights, position, want_y, d_weights, d_y, stream)
