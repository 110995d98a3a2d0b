"""Behind the router: selection, balance and the experts' products in 8-bit integers (argument marshalling only).

    m.apply_router(logits)                                          # steer (a Mix context), then, without a context:
    idx, weights = mix.router_topk(logits, k)                       # the experts of each token
    offsets, order, position = mix.expert_order(idx, n_experts)     # the tokens by expert
    codes, scale = mix.quantize_rows(hidden, order=order, k=k)      # 8-bit rows, each expert's next to each other
    y = mix.linear_int_grouped(codes, scale, W, w_scale, offsets)   # each expert's product
    out = mix.expert_combine(y, weights, position)                  # summed over each token's experts
    loss, counts, mean_p, rows = mix.router_balance(logits, idx, seg)   # what the steering did to each request's load

Every function works on the device of its tensors, on the stream given or that device's current one.  Outputs that are not given
are allocated by torch on that device's current stream; with a stream of your own, give the outputs, or make that stream current.
The C ABI (include/mix.h) states the arithmetic.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as B
from .binding import MIX_ACT_SIGMOID, MIX_ACT_SOFTMAX, MixError  # noqa: F401

_DTYPE = {torch.float32: B.MIX_DTYPE_F32, torch.bfloat16: B.MIX_DTYPE_BF16, torch.float16: B.MIX_DTYPE_F16}
_ERR_LEN = 256


def _call(device, fn, args, stream):
    """fn(*args, stream, errbuf, errbuf_len) with `device` current."""
    here = torch._C._cuda_getDevice()
    if device.index != here:
        with torch.cuda.device(device):
            return _call(device, fn, args, stream)
    err = C.create_string_buffer(_ERR_LEN)
    rc = fn(*args, B._stream(stream), err, _ERR_LEN)
    if rc != 0:
        raise MixError(rc, err.value.decode())


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _tensor(t, name, dtypes, dim, like=None):
    _need(isinstance(t, torch.Tensor) and t.is_cuda, "%s must be a CUDA tensor" % name)
    _need(t.dtype in dtypes if isinstance(dtypes, (tuple, dict)) else t.dtype == dtypes, "%s has type %s" % (name, t.dtype))
    _need(t.dim() == dim, "%s must have %d dimensions, not %d" % (name, dim, t.dim()))
    _need(all(n < 2**31 for n in t.shape), "%s is too large" % name)
    _need(like is None or t.device == like.device, "%s is on another device" % name)
    return t


def _rows(t, name, dtypes, like=None):
    """A matrix whose rows may lie apart: (pointer, row stride)."""
    _tensor(t, name, dtypes, 2, like)
    _need(t.shape[1] <= 1 or t.stride(1) == 1, "%s: the elements of a row must lie next to each other" % name)
    return t.data_ptr(), (t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1))


def _dense(t, name, dtype, shape, like):
    """A tensor without gaps, of one shape: its pointer."""
    _tensor(t, name, dtype, len(shape), like)
    _need(tuple(t.shape) == tuple(shape), "%s has shape %s, not %s" % (name, tuple(t.shape), tuple(shape)))
    _need(t.is_contiguous(), "%s must be contiguous" % name)
    return t.data_ptr()


def _workspace(n, device):
    if n < 0:
        raise MixError(int(n), "the sizes are out of range")
    return torch.empty(max(int(n), 1), dtype=torch.uint8, device=device)


def router_topk(logits, k, act=MIX_ACT_SOFTMAX, renormalise=True, n_live=None, idx=None, weights=None, stream=None):
    """The k largest logits of each row -> idx int32 [T, k] (largest first, of equal ones the lower index first) and weights
    fp32 [T, k]: their softmax or sigmoid values, divided by their sum where `renormalise`.  logits: fp32, bf16 or fp16
    [T, n_experts].  -inf and NaN are never chosen (-1, weight 0, where fewer than k are left), +inf shares the row.  n_live: int32[1]
    on the device; rows from there on are padding and get -1 and 0."""
    lib = B.load_library()
    ptr, ld = _rows(logits, "logits", _DTYPE)
    T, E = logits.shape
    dev = logits.device
    _need(0 < int(k) <= E, "k is %d of %d experts" % (int(k), E))
    live = None if n_live is None else _dense(n_live, "n_live", torch.int32, (1,), logits)
    idx = torch.empty((T, int(k)), dtype=torch.int32, device=dev) if idx is None else idx
    weights = torch.empty((T, int(k)), dtype=torch.float32, device=dev) if weights is None else weights
    _call(dev, lib.mix_router_topk,
          (ptr, _DTYPE[logits.dtype], ld, T, E, int(k), int(act), int(bool(renormalise)), live,
           _dense(idx, "idx", torch.int32, (T, int(k)), logits), _dense(weights, "weights", torch.float32, (T, int(k)), logits)), stream)
    return idx, weights


def router_topk_grad(logits, idx, weights, d_weights, act=MIX_ACT_SOFTMAX, renormalise=True, d_logits=None, stream=None):
    """Gradient of router_topk's weights with respect to the logits: d_logits [T, n_experts] in the logits' type."""
    lib = B.load_library()
    ptr, ld = _rows(logits, "logits", _DTYPE)
    T, E = logits.shape
    _tensor(idx, "idx", torch.int32, 2, logits)
    k = idx.shape[1]
    d_logits = torch.empty((T, E), dtype=logits.dtype, device=logits.device) if d_logits is None else d_logits
    _need(d_logits.shape == logits.shape and d_logits.dtype == logits.dtype, "d_logits must have the logits' shape and type")
    out, ld_d = _rows(d_logits, "d_logits", _DTYPE, logits)
    _call(logits.device, lib.mix_router_topk_grad,
          (ptr, _DTYPE[logits.dtype], ld, T, E, k, int(act), int(bool(renormalise)), _dense(idx, "idx", torch.int32, (T, k), logits),
           _dense(weights, "weights", torch.float32, (T, k), logits), _dense(d_weights, "d_weights", torch.float32, (T, k), logits),
           out, ld_d), stream)
    return d_logits


def expert_order(idx, n_experts, offsets=None, order=None, position=None, stream=None):
    """The entries of idx int32 [T, k] sorted by expert, stably -> offsets int32 [n_experts + 1], order int32 [T * k] (entries
    t * k + j, -1 behind the last), position int32 [T, k] (the entry's place in `order`, -1 where it names no expert)."""
    lib = B.load_library()
    _tensor(idx, "idx", torch.int32, 2)
    n, dev = idx.numel(), idx.device
    _need(0 < int(n_experts) < 2**31, "n_experts is %d" % int(n_experts))
    ws = lib.mix_expert_order_workspace(n, int(n_experts))
    ws = _workspace(ws, dev) if ws != 0 else None
    offsets = torch.empty(int(n_experts) + 1, dtype=torch.int32, device=dev) if offsets is None else offsets
    order = torch.empty(n, dtype=torch.int32, device=dev) if order is None else order
    position = torch.empty(idx.shape, dtype=torch.int32, device=dev) if position is None else position
    _call(dev, lib.mix_expert_order,
          (_dense(idx, "idx", torch.int32, idx.shape, idx), n, int(n_experts), _dense(offsets, "offsets", torch.int32, (int(n_experts) + 1,), idx),
           _dense(order, "order", torch.int32, (n,), idx), _dense(position, "position", torch.int32, idx.shape, idx),
           None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel()), stream)
    _hold(ws, stream)
    return offsets, order, position


def _hold(ws, stream):
    """Scratch memory goes back to torch's allocator on return: where the call went to another stream, only once that has used it."""
    if ws is not None and stream is not None:
        s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream), device=ws.device)
        ws.record_stream(s)


def _segments(seg, like):
    if seg is None:
        return None, 1
    _tensor(seg, "seg", torch.int32, 1, like)
    _need(seg.is_contiguous() and seg.numel() >= 2, "seg must hold the offsets of at least one segment, next to each other")
    return seg.data_ptr(), seg.numel() - 1


def router_balance(logits, idx, seg=None, act=MIX_ACT_SOFTMAX, stream=None):
    """Per segment of rows (seg int32 [n + 1], offsets on the device; None: all rows are one segment): the balance loss fp32 [n], how
    often each expert was chosen int32 [n, n_experts], the experts' mean probabilities fp32 [n, n_experts] and the rows counted
    int32 [n].  idx int32 [T, k] as from router_topk; rows that name no expert do not count."""
    lib = B.load_library()
    ptr, ld = _rows(logits, "logits", _DTYPE)
    T, E = logits.shape
    dev = logits.device
    _tensor(idx, "idx", torch.int32, 2, logits)
    k = idx.shape[1]
    seg_ptr, n = _segments(seg, logits)
    loss = torch.empty(n, dtype=torch.float32, device=dev)
    counts = torch.empty((n, E), dtype=torch.int32, device=dev)
    mean_p = torch.empty((n, E), dtype=torch.float32, device=dev)
    rows = torch.empty(n, dtype=torch.int32, device=dev)
    ws = _workspace(lib.mix_router_balance_workspace(T, E, n), dev)
    _call(dev, lib.mix_router_balance,
          (ptr, _DTYPE[logits.dtype], ld, _dense(idx, "idx", torch.int32, (T, k), logits), T, E, k, int(act), seg_ptr, n, loss.data_ptr(),
           counts.data_ptr(), mean_p.data_ptr(), rows.data_ptr(), ws.data_ptr(), ws.numel()), stream)
    _hold(ws, stream)
    return loss, counts, mean_p, rows


def router_balance_grad(logits, idx, counts, rows, d_loss, seg=None, act=MIX_ACT_SOFTMAX, d_logits=None, stream=None):
    """Gradient of router_balance's losses with respect to the logits, for d_loss fp32 [n] and the counts and rows that it gave."""
    lib = B.load_library()
    ptr, ld = _rows(logits, "logits", _DTYPE)
    T, E = logits.shape
    _tensor(idx, "idx", torch.int32, 2, logits)
    k = idx.shape[1]
    seg_ptr, n = _segments(seg, logits)
    d_logits = torch.empty((T, E), dtype=logits.dtype, device=logits.device) if d_logits is None else d_logits
    _need(d_logits.shape == logits.shape and d_logits.dtype == logits.dtype, "d_logits must have the logits' shape and type")
    out, ld_d = _rows(d_logits, "d_logits", _DTYPE, logits)
    _call(logits.device, lib.mix_router_balance_grad,
          (ptr, _DTYPE[logits.dtype], ld, _dense(idx, "idx", torch.int32, (T, k), logits), T, E, k, int(act), seg_ptr, n,
           _dense(counts, "counts", torch.int32, (n, E), logits), _dense(rows, "rows", torch.int32, (n,), logits),
           _dense(d_loss, "d_loss", torch.float32, (n,), logits), out, ld_d), stream)
    return d_logits


def quantize_rows(x, order=None, k=1, codes=None, scale=None, stream=None):
    """Rows of x (bf16 or fp16 [T, d], d a multiple of 16) as 8-bit integers: codes int8 [n, d] and scale fp32 [n], codes * scale being
    the nearest to x.  With `order` (expert_order's, int32 [n]) row i is row order[i] // k of x; entries of -1 give zeros."""
    lib = B.load_library()
    ptr, ld = _rows(x, "x", (torch.bfloat16, torch.float16))
    T, d = x.shape
    if order is not None:
        _tensor(order, "order", torch.int32, 1, x)
    n = T if order is None else order.numel()
    codes = torch.empty((n, d), dtype=torch.int8, device=x.device) if codes is None else codes
    scale = torch.empty(n, dtype=torch.float32, device=x.device) if scale is None else scale
    _call(x.device, lib.mix_quantize_rows,
          (ptr, _DTYPE[x.dtype], ld, T, None if order is None else _dense(order, "order", torch.int32, (n,), x), int(k), n, d,
           _dense(codes, "codes", torch.int8, (n, d), x), _dense(scale, "scale", torch.float32, (n,), x)), stream)
    return codes, scale


def linear_int(codes, scale, W, w_scale, bias=None, out=None, dtype=torch.bfloat16, stream=None):
    """out[t, n] = (codes[t] . W[n]) scale[t] w_scale[n] + bias[n], the product of 8-bit integers exact, in `dtype` (or out's type).
    codes int8 [T, K], scale fp32 [T]; W int8 [N, K], w_scale fp32 [N], bias fp32 [N]."""
    lib = B.load_library()
    _tensor(codes, "codes", torch.int8, 2)
    _tensor(W, "W", torch.int8, 2, codes)
    (T, K), N = codes.shape, W.shape[0]
    out = torch.empty((T, N), dtype=dtype, device=codes.device) if out is None else out
    optr, ld = _rows(out, "out", _DTYPE, codes)
    _need(tuple(out.shape) == (T, N), "out has shape %s, not %s" % (tuple(out.shape), (T, N)))
    _call(codes.device, lib.mix_linear_int,
          (_dense(codes, "codes", torch.int8, (T, K), codes), _dense(scale, "scale", torch.float32, (T,), codes), T, K,
           _dense(W, "W", torch.int8, (N, K), codes), _dense(w_scale, "w_scale", torch.float32, (N,), codes), N,
           None if bias is None else _dense(bias, "bias", torch.float32, (N,), codes), optr, _DTYPE[out.dtype], ld), stream)
    return out


def linear_int_grouped(codes, scale, W, w_scale, offsets, bias=None, out=None, dtype=torch.bfloat16, stream=None):
    """linear_int with a weight set per group of rows: rows offsets[e] .. offsets[e + 1) of codes (int8 [n, K]) go through W[e]
    (int8 [n_experts, N, K]; w_scale and bias fp32 [n_experts, N]).  Rows of `out` that belong to no expert are left as they were."""
    lib = B.load_library()
    _tensor(codes, "codes", torch.int8, 2)
    _tensor(W, "W", torch.int8, 3, codes)
    (n, K), (E, N) = codes.shape, W.shape[:2]
    out = torch.empty((n, N), dtype=dtype, device=codes.device) if out is None else out
    optr, ld = _rows(out, "out", _DTYPE, codes)
    _need(tuple(out.shape) == (n, N), "out has shape %s, not %s" % (tuple(out.shape), (n, N)))
    _call(codes.device, lib.mix_linear_int_grouped,
          (_dense(codes, "codes", torch.int8, (n, K), codes), _dense(scale, "scale", torch.float32, (n,), codes), n, K,
           _dense(W, "W", torch.int8, (E, N, K), codes), _dense(w_scale, "w_scale", torch.float32, (E, N), codes), E, N,
           _dense(offsets, "offsets", torch.int32, (E + 1,), codes),
           None if bias is None else _dense(bias, "bias", torch.float32, (E, N), codes), optr, _DTYPE[out.dtype], ld), stream)
    return out


def linear_int_status(stream=None) -> int:
    """The status bits of the 8-bit products on the current device since the last call (MIX_STATUS_WAIT_TIMEOUT or 0); synchronises."""
    bits = C.c_uint(0)
    _call(torch.device("cuda", torch._C._cuda_getDevice()), B.load_library().mix_linear_int_status, (C.byref(bits),), stream)
    return int(bits.value)


def expert_combine(y, weights, position, out=None, stream=None):
    """out[t] = sum_j weights[t, j] y[position[t, j]] -> [T, N] in y's type.  y [n, N] in expert_order's order; entries of -1 do not count."""
    lib = B.load_library()
    yptr, ld_y = _rows(y, "y", _DTYPE)
    _tensor(position, "position", torch.int32, 2, y)
    (n, N), (T, k) = y.shape, position.shape
    out = torch.empty((T, N), dtype=y.dtype, device=y.device) if out is None else out
    _need(tuple(out.shape) == (T, N) and out.dtype == y.dtype, "out must be [T, N] in y's type")
    optr, ld = _rows(out, "out", _DTYPE, y)
    _call(y.device, lib.mix_expert_combine,
          (yptr, _DTYPE[y.dtype], ld_y, n, _dense(weights, "weights", torch.float32, (T, k), y),
           _dense(position, "position", torch.int32, (T, k), y), T, k, N, optr, ld), stream)
    return out
