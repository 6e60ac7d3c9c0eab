"""Operators around a policy net (include/reuse_ops.h): layer norm, the gated
delta rule's memory and the sampling of actions; the norm of a residual stream,
the short convolution, the selective scan and the log-probabilities of actions
that were taken, on torch tensors.

Every function only checks its arguments, allocates what the caller did not
give and passes pointers on: the work runs in the library's HIP kernels, on
``stream`` (the current stream by default).  There is no fallback.  float32 and
bfloat16 data are taken; statistics, memories, settings and the gradients of
float32 arguments are float32.

With ``stream`` a call does what it does under ``torch.cuda.stream(stream)``:
results and scratch are that stream's memory, whose reuse is ordered on it.  As
there, the caller orders the streams that write the arguments and read the
results, and records (``Tensor.record_stream``) a tensor that another stream
still uses when it is dropped.

Nothing is recorded for autograd: where it is on, tensors that require grad are
refused.  Call under ``torch.no_grad()``, or in a ``torch.autograd.Function``
whose backward makes the ``_backward`` call (examples/recurrent_policy.py).

A policy that remembers, one frame of n streams at a time:

    x = layer_norm(features, w, b)
    q, k, v, g, beta = ...                       # the caller's projections of x
    h = delta_step(q, k, v, g, beta, memory)     # memory: [streams][heads][dk][dv], in place
    actions, logprobs = sample(logits, u)        # logits: the caller's projection of h

and over whole episodes ``delta_forward(..., save=True)`` with
``delta_backward`` and ``layer_norm_backward`` for the gradients.

One whose memory is a window and a state, in a block beside a residual stream x:

    u, z, dt, b, c = ...                         # the caller's projections of rms_norm(x, w)
    u = causal_conv_step(u, w_conv, window)      # [streams][taps - 1][channels], in place
    h = scan_step(u, dt, a, b, c, state, z=z)    # [streams][channels][states], in place
    y, x = rms_norm(h @ w_mid, w, residual=x)    # for the next block, or for logits

and over whole episodes ``causal_conv``, ``scan_forward(..., save=True)`` and
``log_probs(logits, actions, with_stats=True)`` with their ``_backward`` calls.
"""
from __future__ import annotations

import ctypes
import operator
from typing import Optional

import torch

from . import binding as B

RN_SAMPLE_MAX_VOCAB = 1 << 20
RN_LOGPROBS_MAX_TOP = 64
RN_CONV_MAX_TAPS = 4
RN_SCAN_MAX_STATES = 64
RN_DELTA_MAX_DIM = 128

# Every entry point include/reuse_ops.h declares.
EXPORTS = (
    "reuse_ops_last_error", "reuse_ops_layer_norm", "reuse_ops_layer_norm_backward_scratch_bytes",
    "reuse_ops_layer_norm_backward", "reuse_ops_sample", "reuse_ops_delta_step", "reuse_ops_delta_saved_bytes",
    "reuse_ops_delta_scratch_bytes", "reuse_ops_delta_backward_scratch_bytes", "reuse_ops_delta_forward",
    "reuse_ops_delta_backward", "reuse_ops_rms_norm", "reuse_ops_rms_norm_backward_scratch_bytes",
    "reuse_ops_rms_norm_backward", "reuse_ops_log_probs_scratch_bytes", "reuse_ops_log_probs",
    "reuse_ops_log_probs_backward", "reuse_ops_causal_conv_step", "reuse_ops_causal_conv",
    "reuse_ops_causal_conv_backward_scratch_bytes", "reuse_ops_causal_conv_backward", "reuse_ops_scan_step",
    "reuse_ops_scan_saved_bytes", "reuse_ops_scan_scratch_bytes", "reuse_ops_scan_backward_scratch_bytes",
    "reuse_ops_scan_forward", "reuse_ops_scan_backward",
)


class rn_sample_params(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_float), ("top_k", ctypes.c_int32), ("top_p", ctypes.c_float),
                ("min_p", ctypes.c_float), ("dev_temperature", ctypes.c_void_p), ("dev_top_k", ctypes.c_void_p),
                ("dev_top_p", ctypes.c_void_p), ("dev_min_p", ctypes.c_void_p)]


class rn_delta_shape(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("heads_k", ctypes.c_int32), ("heads_v", ctypes.c_int32),
                ("dk", ctypes.c_int32), ("dv", ctypes.c_int32), ("tokens", ctypes.c_int64), ("dtype", ctypes.c_int),
                ("scale", ctypes.c_float), ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64),
                ("v_stride", ctypes.c_int64), ("even", ctypes.c_int32)]


class rn_conv_shape(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("channels", ctypes.c_int32), ("taps", ctypes.c_int32),
                ("tokens", ctypes.c_int64), ("dtype", ctypes.c_int), ("silu", ctypes.c_int32),
                ("x_stride", ctypes.c_int64)]


class rn_scan_shape(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("channels", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("states", ctypes.c_int32), ("tokens", ctypes.c_int64), ("dtype", ctypes.c_int),
                ("softplus", ctypes.c_int32), ("u_stride", ctypes.c_int64), ("dt_stride", ctypes.c_int64),
                ("b_stride", ctypes.c_int64), ("c_stride", ctypes.c_int64), ("z_stride", ctypes.c_int64)]


class rn_scan_inputs(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("u", "dt", "b", "c", "a", "d", "z", "dt_bias")]


class rn_scan_grads(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("du", "ddt", "db", "dc", "dz", "da", "dd", "ddt_bias", "dstate")]


_ops = None


def load_ops():
    """The library with the operators' C signatures declared.  Raises if it is not built."""
    global _ops
    if _ops is not None:
        return _ops
    L = B.load_library()
    P, I32, I64, SZ, F, st = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float,
                              ctypes.c_int)
    shape, conv = ctypes.POINTER(rn_delta_shape), ctypes.POINTER(rn_conv_shape)
    scan, given = ctypes.POINTER(rn_scan_shape), ctypes.POINTER(rn_scan_inputs)
    for name, res, args in (
            ("last_error", ctypes.c_char_p, []),
            ("layer_norm", st, [I64, I32, P, I64, st, P, P, F, P, I64, P, P]),
            ("layer_norm_backward_scratch_bytes", SZ, [I64, I32]),
            ("layer_norm_backward", st, [I64, I32, P, I64, P, I64, st, P, P, P, I64, P, P, I32, P, SZ, P]),
            ("rms_norm", st, [I64, I32, P, I64, st, P, I64, P, F, P, P, P, P, P, P]),
            ("rms_norm_backward_scratch_bytes", SZ, [I64, I32]),
            ("rms_norm_backward", st, [I64, I32, P, I64, P, I64, st, P, P, P, I64, P, P, I32, P, SZ, P]),
            ("sample", st, [I32, I32, P, I64, st, P, ctypes.POINTER(rn_sample_params), P, P, P]),
            ("log_probs_scratch_bytes", SZ, [I32, I32, I32]),
            ("log_probs", st, [I32, I32, P, I64, st, P, F, I32, P, P, P, P, P, P, SZ, P]),
            ("log_probs_backward", st, [I32, I32, P, I64, st, P, F, P, P, P, P, I64, P]),
            ("causal_conv_step", st, [conv, P, P, P, P, I32, P, P, P]),
            ("causal_conv", st, [conv, P, P, P, P, P, P, P, P]),
            ("causal_conv_backward_scratch_bytes", SZ, [conv]),
            ("causal_conv_backward", st, [conv, P, P, P, P, P, P, P, P, P, P, P, P, SZ, P]),
            ("scan_step", st, [scan, given, P, I32, P, P, P]),
            ("scan_saved_bytes", SZ, [scan]),
            ("scan_scratch_bytes", SZ, [scan]),
            ("scan_backward_scratch_bytes", SZ, [scan]),
            ("scan_forward", st, [scan, given, P, P, P, P, P, SZ, P, SZ, P]),
            ("scan_backward", st, [scan, given, P, P, SZ, P, P, ctypes.POINTER(rn_scan_grads), P, SZ, P]),
            ("delta_step", st, [shape, P, P, P, P, P, P, I32, P, P, P]),
            ("delta_saved_bytes", SZ, [shape]),
            ("delta_scratch_bytes", SZ, [shape]),
            ("delta_backward_scratch_bytes", SZ, [shape]),
            ("delta_forward", st, [shape, P, P, P, P, P, P, P, P, P, P, SZ, P, SZ, P]),
            ("delta_backward", st, [shape, P, P, P, P, P, P, P, SZ, P, P, P, P, P, P, P, P, P, SZ, P])):
        f = getattr(L, "reuse_ops_" + name)
        f.restype, f.argtypes = res, args
    _ops = L
    return L


def reuse_ops_last_error() -> str:
    return load_ops().reuse_ops_last_error().decode()


def _check(status: int) -> None:
    if status != B.RN_OK:
        raise B.ReuseNetError(status, reuse_ops_last_error())


_F32, _BF16, _I32, _F8 = torch.float32, torch.bfloat16, torch.int32, torch.float8_e4m3fn
_CODES = {_F32: B.RN_F32, _BF16: B.RN_BF16}


# The C ABI takes raw pointers and sizes: whatever does not match what the
# kernels will read or write is refused here, before any launch.
def _data(x, what: str) -> int:
    """The dtype code of a float32 or bfloat16 tensor on a GPU."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    code = _CODES.get(x.dtype)
    if code is None:
        raise TypeError(f"{what} must be float32 or bfloat16, got {x.dtype}")
    if not x.is_cuda:
        raise ValueError(f"{what} must be on a GPU, got {x.device}")
    return code


def _like(x, what: str, dtype, device, shape) -> int:
    """The pointer of a contiguous tensor that has to be just so."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    if x.dtype is dtype and x.device == device and x.shape == shape and x.is_contiguous():
        return x.data_ptr()
    if x.dtype is not dtype:
        raise TypeError(f"{what} must be {dtype}, got {x.dtype}")
    if x.device != device:
        raise ValueError(f"{what} must be on {device}, got {x.device}")
    if x.shape != shape:
        raise ValueError(f"{what} must have shape {tuple(shape)}, got {tuple(x.shape)}")
    raise ValueError(f"{what} must be contiguous")


def _opt(x, what: str, dtype, device, shape) -> Optional[int]:
    return None if x is None else _like(x, what, dtype, device, shape)


def _count(v: int, what: str) -> int:
    """v as the C calls' 32-bit counts hold it: ctypes drops what is above them without a word."""
    if v > 0x7fffffff:
        raise ValueError(f"{what} must be below 2^31, got {v}")
    return v


def _rows(x, what: str):
    """(rows, row stride) of a tensor read as rows of its last axis."""
    width = x.shape[-1]
    if x.is_contiguous():
        return x.numel() // max(1, width), width
    if x.dim() == 2 and x.stride(1) == 1 and (x.stride(0) >= width or x.shape[0] <= 1):
        return x.shape[0], x.stride(0)
    if width == 1 or x.stride(-1) == 1:
        # Leading axes that fold into one: each strides over the whole of the next.
        lead = [(n, s) for n, s in zip(x.shape[:-1], x.stride()[:-1]) if n != 1]
        if all(a[1] == b[0] * b[1] for a, b in zip(lead, lead[1:])) and (not lead or lead[-1][1] >= width):
            rows = 1
            for n, _ in lead:
                rows *= n
            return rows, (lead[-1][1] if lead else width)
    raise ValueError(f"{what} must have contiguous rows at one stride, got strides {x.stride()}")


# The small calls' time is the host's: the current stream's handle without a
# Stream object around it, where torch has that (1.9 -> 0.1 us).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _no_grad(*tensors) -> None:
    """Refuses what autograd would have to follow through a call that it does not see."""
    if torch.is_grad_enabled():
        for x in tensors:
            if getattr(x, "requires_grad", False):
                raise ValueError("a tensor requires grad, which is not recorded here: call under torch.no_grad(), "
                                 "or in a torch.autograd.Function with the backward call")


def _on(stream, x):
    """`stream` as the current one, for the memory a call makes as well as for its launches."""
    if isinstance(x, torch.Tensor) and x.is_cuda and x.device != stream.device:
        raise ValueError(f"stream is on {stream.device}, the tensors are on {x.device}")
    return torch.cuda.stream(stream)


def _launch(device, call, *args) -> None:
    """The call on the current stream, with the tensors' GPU current."""
    index = device.index
    s = _raw_stream(index)
    if torch.cuda.current_device() == index:
        status = call(*args, s)
    else:
        with torch.cuda.device(device):
            status = call(*args, s)
    if status:
        raise B.ReuseNetError(status, reuse_ops_last_error())


def _empty(like, shape=None, dtype=None):
    """A contiguous tensor of `like`'s device (and shape and dtype)."""
    if shape is None:
        return torch.empty_like(like, memory_format=torch.contiguous_format)
    return like.new_empty(shape, dtype=dtype)


# ------------------------------------------------------------------ layer norm

def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, with_stats: bool = False, out=None, stream=None):
    """Layer norm over the last axis (reuse_ops_layer_norm).

    x: [..., width] float32 or bfloat16, rows contiguous and at one stride;
    weight, bias: [width] float32 or None.  Returns y in x's dtype, and with
    with_stats also the [rows][2] float32 mean and 1/sd for the backward call.
    """
    if stream is not None:
        with _on(stream, x):
            return layer_norm(x, weight, bias, eps, with_stats, out)
    _no_grad(x, weight, bias)
    code = _data(x, "x")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must have a last axis of 1 or more")
    dev, width = x.device, _count(x.shape[-1], "width")
    rows, stride = _rows(x, "x")
    w = None if weight is None else _like(weight, "weight", _F32, dev, (width,))
    b = None if bias is None else _like(bias, "bias", _F32, dev, (width,))
    if out is None:
        out = _empty(x)
        y = out.data_ptr()
    else:
        y = _like(out, "out", x.dtype, dev, x.shape)
    stats = _empty(x, (rows, 2), _F32) if with_stats else None
    _launch(dev, load_ops().reuse_ops_layer_norm, rows, width, x.data_ptr(), stride, code, w, b, eps, y, width,
            None if stats is None else stats.data_ptr())
    return (out, stats) if with_stats else out


def layer_norm_backward(dy, x, weight, stats, dx=None, dweight=None, dbias=None, accumulate: bool = False,
                        want_params: bool = True, stream=None):
    """(dx, dweight, dbias) of layer_norm (reuse_ops_layer_norm_backward).

    stats: from the forward call.  dweight, dbias: [width] float32 buffers to
    write, or to add to with accumulate; made here if None.  want_params =
    False: dx only, the other two are returned as given.
    """
    if stream is not None:
        with _on(stream, x):
            return layer_norm_backward(dy, x, weight, stats, dx, dweight, dbias, accumulate, want_params)
    _no_grad(dy, x, weight, stats)
    code = _data(x, "x")
    if not isinstance(dy, torch.Tensor) or dy.dtype is not x.dtype or dy.shape != x.shape or dy.device != x.device:
        raise ValueError("dy must have x's dtype, shape and device")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must have a last axis of 1 or more")
    dev, width = x.device, _count(x.shape[-1], "width")
    rows, xs = _rows(x, "x")
    _, dys = _rows(dy, "dy")
    w = _opt(weight, "weight", _F32, dev, (width,))
    st = _like(stats, "stats", _F32, dev, (rows, 2))
    if dx is None:
        dx = _empty(x)
        d = dx.data_ptr()
    else:
        d = _like(dx, "dx", x.dtype, dev, x.shape)
    L = load_ops()
    dw = db = sc = None
    need = 0
    if want_params:
        if accumulate and (dweight is None or dbias is None):
            raise ValueError("accumulate needs dweight and dbias")
        if dweight is None:
            dweight = _empty(x, width, _F32)
        if dbias is None:
            dbias = _empty(x, width, _F32)
        dw = _like(dweight, "dweight", _F32, dev, (width,))
        db = _like(dbias, "dbias", _F32, dev, (width,))
        need = L.reuse_ops_layer_norm_backward_scratch_bytes(rows, width)
        scratch = _empty(x, need, torch.uint8)
        sc = scratch.data_ptr()
    _launch(dev, L.reuse_ops_layer_norm_backward, rows, width, dy.data_ptr(), dys, x.data_ptr(), xs, code, w,
            st, d, width, dw, db, int(accumulate), sc, need)
    return dx, dweight, dbias


# ------------------------------------------------------------------ residual norm

def _same(x, like, what: str, of: str) -> None:
    """x has the dtype, shape and device of `like`."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    if x.dtype is not like.dtype or x.shape != like.shape or x.device != like.device:
        raise ValueError(f"{what} must have {of}'s dtype, shape and device")


def rms_norm(x, weight=None, residual=None, eps: float = 1e-5, with_stats: bool = False, quantize: bool = False,
             out=None, scales=None, total=None, stream=None):
    """Norm by the root mean square over the last axis, of x or of x + residual (reuse_ops_rms_norm).

    x, residual: [..., width] float32 or bfloat16, rows contiguous and at one
    stride; weight: [width] float32 or None.  Returns y in x's dtype; with
    quantize in its place y / scales as float8_e4m3fn and the [rows] float32
    scales; then x + residual in x's dtype if there is a residual, and with
    with_stats the [rows] float32 1/rms for the backward call.  One result
    comes alone, more as a tuple.  out, total: where y and the sum go (they
    may be x or the residual); made here if None.
    """
    if stream is not None:
        with _on(stream, x):
            return rms_norm(x, weight, residual, eps, with_stats, quantize, out, scales, total)
    _no_grad(x, weight, residual)
    code = _data(x, "x")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("x must have a last axis of 1 or more")
    dev, width = x.device, _count(x.shape[-1], "width")
    rows, stride = _rows(x, "x")
    w = None if weight is None else _like(weight, "weight", _F32, dev, (width,))
    r, rs, tp = None, 0, None
    if residual is not None:
        _same(residual, x, "residual", "x")
        r, rs = residual.data_ptr(), _rows(residual, "residual")[1]
        if total is None:
            total = _empty(x)
        tp = _like(total, "total", x.dtype, dev, x.shape)
    elif total is not None:
        raise ValueError("without a residual there is no total")
    if out is None:
        out = _empty(x, x.shape, _F8) if quantize else _empty(x)
    o = _like(out, "out", _F8 if quantize else x.dtype, dev, x.shape)
    got, sp = [out], None
    if quantize:
        if scales is None:
            scales = _empty(x, rows, _F32)
        sp = _like(scales, "scales", _F32, dev, (rows,))
        got.append(scales)
    elif scales is not None:
        raise ValueError("scales are written with quantize only")
    if residual is not None:
        got.append(total)
    stats = None
    if with_stats:
        stats = _empty(x, rows, _F32)
        got.append(stats)
    _launch(dev, load_ops().reuse_ops_rms_norm, rows, width, x.data_ptr(), stride, code, r, rs, w, eps,
            None if quantize else o, o if quantize else None, sp, tp, None if stats is None else stats.data_ptr())
    return got[0] if len(got) == 1 else tuple(got)


def rms_norm_backward(dy, total, weight, stats, dtotal=None, dx=None, dweight=None, accumulate: bool = False,
                      want_params: bool = True, stream=None):
    """(dx, dweight) of rms_norm (reuse_ops_rms_norm_backward); dx is the residual's gradient too.

    total, stats: from the forward call (x itself if it had no residual).
    dtotal: the gradient that reaches the sum by another way, or None.
    dweight: [width] float32 buffer to write, or to add to with accumulate;
    made here if None.  want_params = False: dx only, dweight is returned as
    given.
    """
    if stream is not None:
        with _on(stream, total):
            return rms_norm_backward(dy, total, weight, stats, dtotal, dx, dweight, accumulate, want_params)
    _no_grad(dy, total, weight, stats, dtotal)
    code = _data(total, "total")
    if total.dim() < 1 or total.shape[-1] < 1:
        raise ValueError("total must have a last axis of 1 or more")
    _same(dy, total, "dy", "total")
    dev, width = total.device, _count(total.shape[-1], "width")
    rows, ts = _rows(total, "total")
    _, dys = _rows(dy, "dy")
    dt, dts = None, 0
    if dtotal is not None:
        _same(dtotal, total, "dtotal", "total")
        dt, dts = dtotal.data_ptr(), _rows(dtotal, "dtotal")[1]
    w = _opt(weight, "weight", _F32, dev, (width,))
    st = _like(stats, "stats", _F32, dev, (rows,))
    if dx is None:
        dx = _empty(total)
    d = _like(dx, "dx", total.dtype, dev, total.shape)
    L = load_ops()
    dw = sc = None
    need = 0
    if want_params:
        if accumulate and dweight is None:
            raise ValueError("accumulate needs dweight")
        if dweight is None:
            dweight = _empty(total, width, _F32)
        dw = _like(dweight, "dweight", _F32, dev, (width,))
        need = L.reuse_ops_rms_norm_backward_scratch_bytes(rows, width)
        scratch = _empty(total, need, torch.uint8)
        sc = scratch.data_ptr()
    _launch(dev, L.reuse_ops_rms_norm_backward, rows, width, dy.data_ptr(), dys, total.data_ptr(), ts, code, w, st,
            dt, dts, d, dw, int(accumulate), sc, need)
    return dx, dweight


# ------------------------------------------------------------------ sampling

def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, tokens=None, logprobs=None, stream=None):
    """Draw one choice per row of logits [n][vocab] (reuse_ops_sample).

    u: [n] float32 random numbers in [0, 1).  temperature, top_p, min_p: a
    number, or [n] float32; top_k: a number, or [n] int32.  Temperature 0 is
    greedy, top_k 0 and top_p 1 leave the filter off.  Returns ([n] int32
    choices, [n] float32 log-probabilities among what the filters left).
    """
    if stream is not None:
        with _on(stream, logits):
            return sample(logits, u, temperature, top_k, top_p, min_p, tokens, logprobs)
    _no_grad(logits)
    code = _data(logits, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits must have shape (n, vocab), got {tuple(logits.shape)}")
    n, vocab = logits.shape
    dev = logits.device
    _count(n, "n")
    if not 1 <= vocab <= RN_SAMPLE_MAX_VOCAB:
        raise ValueError(f"vocab must be 1..{RN_SAMPLE_MAX_VOCAB}, got {vocab}")
    rows, stride = _rows(logits, "logits")
    up = _like(u, "u", _F32, dev, (n,))
    def setting(value, name, dtype):
        """(number, pointer): one of the two is what counts."""
        if isinstance(value, torch.Tensor):
            return 0, _like(value, name, dtype, dev, (n,))
        return value, None

    t, tp = setting(temperature, "temperature", _F32)
    k, kp = setting(top_k, "top_k", _I32)
    k = min(max(operator.index(k), 0), RN_SAMPLE_MAX_VOCAB)     # above the vocabulary and below 1: all
    p, pp = setting(top_p, "top_p", _F32)
    m, mp = setting(min_p, "min_p", _F32)
    params = rn_sample_params(t, k, p, m, tp, kp, pp, mp)
    if tokens is None:
        tokens = _empty(logits, n, _I32)
    if logprobs is None:
        logprobs = _empty(logits, n, _F32)
    ids = _like(tokens, "tokens", _I32, dev, (n,))
    lp = _like(logprobs, "logprobs", _F32, dev, (n,))
    _launch(dev, load_ops().reuse_ops_sample, n, vocab, logits.data_ptr(), stride, code, up,
            ctypes.byref(params), ids, lp)
    return tokens, logprobs


# ------------------------------------------------------------------ log-probabilities

def _choices(logits, tokens):
    """(dtype code, n, vocab, row stride, the choices' pointer) of a row of logits and a choice each."""
    code = _data(logits, "logits")
    if logits.dim() != 2:
        raise ValueError(f"logits must have shape (n, vocab), got {tuple(logits.shape)}")
    n, vocab = logits.shape
    _count(n, "n")
    if not 1 <= vocab <= RN_SAMPLE_MAX_VOCAB:
        raise ValueError(f"vocab must be 1..{RN_SAMPLE_MAX_VOCAB}, got {vocab}")
    return code, n, vocab, _rows(logits, "logits")[1], _like(tokens, "tokens", _I32, logits.device, (n,))


def log_probs(logits, tokens, temperature: float = 1.0, top: int = 0, with_stats: bool = False, stream=None):
    """Log-probabilities of given choices, and the entropy of their rows (reuse_ops_log_probs).

    logits: [n][vocab] float32 or bfloat16, tokens: [n] int32 choices; one
    outside 0..vocab-1 has log-probability 0 and no gradient.  temperature: a
    number above 0.  Returns ([n], [n]) float32; with top also the [n][top]
    int32 likeliest choices and their float32 log-probabilities, from the
    likeliest down; with with_stats also the [n][4] float32 that
    log_probs_backward reads.
    """
    if stream is not None:
        with _on(stream, logits):
            return log_probs(logits, tokens, temperature, top, with_stats)
    _no_grad(logits)
    code, n, vocab, stride, ids = _choices(logits, tokens)
    top = operator.index(top)
    if not 0 <= top <= min(vocab, RN_LOGPROBS_MAX_TOP):
        raise ValueError(f"top must be 0..{min(vocab, RN_LOGPROBS_MAX_TOP)}, got {top}")
    L = load_ops()
    need = L.reuse_ops_log_probs_scratch_bytes(n, vocab, top)
    scratch = _empty(logits, need, torch.uint8)
    got = [_empty(logits, n, _F32), _empty(logits, n, _F32)]
    if top:
        got += [_empty(logits, (n, top), _I32), _empty(logits, (n, top), _F32)]
    if with_stats:
        got.append(_empty(logits, (n, 4), _F32))
    _launch(logits.device, L.reuse_ops_log_probs, n, vocab, logits.data_ptr(), stride, code, ids, temperature, top,
            got[0].data_ptr(), got[1].data_ptr(), got[2].data_ptr() if top else None,
            got[3].data_ptr() if top else None, got[-1].data_ptr() if with_stats else None, scratch.data_ptr(), need)
    return tuple(got)


def log_probs_backward(dlogprobs, dentropy, logits, tokens, stats, temperature: float = 1.0, dlogits=None, stream=None):
    """dlogits of log_probs (reuse_ops_log_probs_backward).

    dlogprobs, dentropy: [n] float32 gradients of the two, or None for 0;
    logits, tokens, temperature: the forward call's, stats its result.
    dlogits: [n][vocab] in logits' dtype, at any row stride; it may be logits
    itself; made here if None.
    """
    if stream is not None:
        with _on(stream, logits):
            return log_probs_backward(dlogprobs, dentropy, logits, tokens, stats, temperature, dlogits)
    _no_grad(dlogprobs, dentropy, logits, stats)
    code, n, vocab, stride, ids = _choices(logits, tokens)
    dev = logits.device
    st = _like(stats, "stats", _F32, dev, (n, 4))
    dp = _opt(dlogprobs, "dlogprobs", _F32, dev, (n,))
    de = _opt(dentropy, "dentropy", _F32, dev, (n,))
    if dlogits is None:
        dlogits = _empty(logits)
    _same(dlogits, logits, "dlogits", "logits")
    _launch(dev, load_ops().reuse_ops_log_probs_backward, n, vocab, logits.data_ptr(), stride, code, ids, temperature,
            st, dp, de, dlogits.data_ptr(), _rows(dlogits, "dlogits")[1])
    return dlogits


# ------------------------------------------------------------------ gated delta rule

def _tokens(x, what: str, dtype, tokens: int, device):
    """(heads, size, token stride) of [tokens][heads][size] data whose heads are contiguous."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    if x.dtype is not dtype or x.device != device:
        raise ValueError(f"{what} must have q's dtype and device")
    if x.dim() != 3 or x.shape[0] != tokens:
        raise ValueError(f"{what} must have shape ({tokens}, heads, size), got {tuple(x.shape)}")
    _, heads, size = x.shape
    if heads < 1 or size < 1:
        raise ValueError(f"{what} must have heads and elements")
    if x.is_contiguous():
        return heads, size, heads * size
    st = x.stride()
    if (size > 1 and st[2] != 1) or (heads > 1 and st[1] != size):
        raise ValueError(f"{what} must be contiguous within a token, got strides {st}")
    if tokens > 1 and st[0] < heads * size:
        raise ValueError(f"{what}: a token's stride is smaller than a token")
    return heads, size, (st[0] if tokens > 1 else heads * size)


def _delta_shape(q, k, v, g, beta, n: int, scale, even: bool = True):
    code = _data(q, "q")
    if q.dim() != 3:
        raise ValueError(f"q must have shape (tokens, heads, dk), got {tuple(q.shape)}")
    tokens, dev, dtype = q.shape[0], q.device, q.dtype
    hk, dk, qs = _tokens(q, "q", dtype, tokens, dev)
    hk2, dk2, ks = _tokens(k, "k", dtype, tokens, dev)
    hv, dv, vs = _tokens(v, "v", dtype, tokens, dev)
    if (hk2, dk2) != (hk, dk):
        raise ValueError("k must have q's shape")
    if hv % hk:
        raise ValueError(f"{hv} value heads cannot share {hk} key heads")
    _count(max(hk, hv, dk, dv, n), "heads, dk, dv and n")
    shape = rn_delta_shape(n, hk, hv, dk, dv, tokens, code, dk ** -0.5 if scale is None else scale, qs, ks, vs, even)
    gp = _like(g, "g", _F32, dev, (tokens, hv))
    bp = _like(beta, "beta", _F32, dev, (tokens, hv))
    return shape, gp, bp, dev, hv, dk, dv


def _sequences(seq_off, n, tokens: int, device):
    """(n, offsets pointer): packed sequences by seq_off, or n even ones."""
    if seq_off is not None:
        if not isinstance(seq_off, torch.Tensor) or seq_off.dim() != 1 or seq_off.shape[0] < 1:
            raise ValueError("seq_off must be a 1-D int32 tensor of n + 1 entries")
        m = seq_off.shape[0] - 1
        if n is not None and n != m:
            raise ValueError(f"n is {n}, seq_off has {m} sequences")
        return m, _like(seq_off, "seq_off", _I32, device, (m + 1,))
    if n is None:
        raise ValueError("give seq_off, or n for even sequences")
    if n < 0 or (n and tokens % n) or (not n and tokens):
        raise ValueError(f"{tokens} tokens are not {n} even sequences")
    return n, None


def delta_step(q, k, v, g, beta, state, stream_ids=None, scale=None, out=None, stream=None):
    """One token for each of n streams, their memories updated in place (reuse_ops_delta_step).

    q, k: [n][heads_k][dk], v: [n][heads_v][dv] float32 or bfloat16; g, beta:
    [n][heads_v] float32; state: [slots][heads_v][dk][dv] float32; stream_ids:
    [n] int32 distinct slots (None: 0..n-1).  scale defaults to dk^-1/2.
    Returns out [n][heads_v][dv].
    """
    if stream is not None:
        with _on(stream, q):
            return delta_step(q, k, v, g, beta, state, stream_ids, scale, out)
    _no_grad(q, k, v, g, beta, state)
    n = q.shape[0] if isinstance(q, torch.Tensor) and q.dim() else 0
    shape, gp, bp, dev, hv, dk, dv = _delta_shape(q, k, v, g, beta, n, scale)
    slots = state.shape[0] if isinstance(state, torch.Tensor) and state.dim() else 0
    sp = _like(state, "state", _F32, dev, (_count(slots, "slots"), hv, dk, dv))
    ids = _opt(stream_ids, "stream_ids", _I32, dev, (n,))
    if ids is None and slots < n:
        raise ValueError(f"{n} streams need as many slots, state has {slots}")
    if out is None:
        out = _empty(v)
    op = _like(out, "out", q.dtype, dev, (n, hv, dv))
    _launch(dev, load_ops().reuse_ops_delta_step, ctypes.byref(shape), q.data_ptr(), k.data_ptr(), v.data_ptr(),
            gp, bp, ids, slots, sp, op)
    return out


def _supported(need: int, call, shape) -> int:
    if need == 0:                                  # re-run the call's own checks to report why
        _check(call(ctypes.byref(shape), *([1] * 5), *([None] * (len(call.argtypes) - 6))))
    return need


def delta_forward(q, k, v, g, beta, seq_off=None, n=None, state=None, final=None, scale=None, save: bool = False,
                  out=None, stream=None):
    """All tokens of n sequences (reuse_ops_delta_forward).

    q, k: [tokens][heads_k][dk], v: [tokens][heads_v][dv], g, beta:
    [tokens][heads_v] float32; sequence i owns tokens seq_off[i] ..
    seq_off[i+1] - 1 (int32, [n + 1]), or n even ones.  state:
    [n][heads_v][dk][dv] float32 first memories (None: zeros); final: where the
    last ones go (made here if None; it may be state).  Returns (out, final),
    with save also the buffer that delta_backward reads.
    """
    if stream is not None:
        with _on(stream, q):
            return delta_forward(q, k, v, g, beta, seq_off, n, state, final, scale, save, out)
    _no_grad(q, k, v, g, beta, state)
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor of shape (tokens, heads, dk)")
    n, off = _sequences(seq_off, n, q.shape[0], q.device)
    shape, gp, bp, dev, hv, dk, dv = _delta_shape(q, k, v, g, beta, n, scale, off is None)
    dims = (n, hv, dk, dv)
    sp = _opt(state, "state", _F32, dev, dims)
    L = load_ops()
    need = _supported(L.reuse_ops_delta_scratch_bytes(ctypes.byref(shape)), L.reuse_ops_delta_forward, shape)
    if final is None:
        final = _empty(q, dims, _F32)
    fp = _like(final, "final", _F32, dev, dims)
    if out is None:
        out = _empty(v)
    op = _like(out, "out", q.dtype, dev, v.shape)
    scratch = _empty(q, need, torch.uint8)
    saved, kept, size = None, None, 0
    if save:
        size = L.reuse_ops_delta_saved_bytes(ctypes.byref(shape))
        saved = _empty(q, size, torch.uint8)
        kept = saved.data_ptr()
    _launch(dev, L.reuse_ops_delta_forward, ctypes.byref(shape), q.data_ptr(), k.data_ptr(), v.data_ptr(), gp,
            bp, off, sp, fp, op, kept, size, scratch.data_ptr(), need)
    return (out, final, saved) if save else (out, final)


def delta_backward(dout, q, k, v, g, beta, seq_off=None, n=None, saved=None, dfinal=None, scale=None,
                   want_dstate: bool = True, stream=None):
    """Gradients (dq, dk, dv, dg, dbeta, dstate) of delta_forward (reuse_ops_delta_backward).

    The inputs are the forward call's, saved its buffer; dout: dJ/dout, dfinal:
    dJ/dfinal or None.  dstate is None without want_dstate.
    """
    if stream is not None:
        with _on(stream, q):
            return delta_backward(dout, q, k, v, g, beta, seq_off, n, saved, dfinal, scale, want_dstate)
    _no_grad(dout, q, k, v, g, beta, dfinal)
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor of shape (tokens, heads, dk)")
    n, off = _sequences(seq_off, n, q.shape[0], q.device)
    shape, gp, bp, dev, hv, dk, dv = _delta_shape(q, k, v, g, beta, n, scale, off is None)
    dims = (n, hv, dk, dv)
    do = _like(dout, "dout", q.dtype, dev, v.shape)
    df = _opt(dfinal, "dfinal", _F32, dev, dims)
    L = load_ops()
    need = _supported(L.reuse_ops_delta_backward_scratch_bytes(ctypes.byref(shape)), L.reuse_ops_delta_backward, shape)
    if not isinstance(saved, torch.Tensor):
        raise TypeError("saved must be the buffer of delta_forward(..., save=True)")
    sp = _like(saved, "saved", torch.uint8, dev, (L.reuse_ops_delta_saved_bytes(ctypes.byref(shape)),))
    gq, gk, gv, dg, dbeta = _empty(q), _empty(k), _empty(v), _empty(g), _empty(beta)
    dstate = _empty(q, dims, _F32) if want_dstate else None
    scratch = _empty(q, need, torch.uint8)
    _launch(dev, L.reuse_ops_delta_backward, ctypes.byref(shape), q.data_ptr(), k.data_ptr(), v.data_ptr(), gp,
            bp, off, sp, saved.numel(), do, df, gq.data_ptr(), gk.data_ptr(), gv.data_ptr(), dg.data_ptr(),
            dbeta.data_ptr(), None if dstate is None else dstate.data_ptr(), scratch.data_ptr(), need)
    return gq, gk, gv, dg, dbeta, dstate


# ------------------------------------------------------------------ short convolution

def _flat(x, what: str, dtype, tokens: int, channels: int, device):
    """(pointer, token stride) of [tokens][channels] data whose channels are contiguous."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    if x.dtype is not dtype or x.device != device:
        raise ValueError(f"{what} must be {dtype} on {device}")
    if x.shape != (tokens, channels):
        raise ValueError(f"{what} must have shape ({tokens}, {channels}), got {tuple(x.shape)}")
    row, one = x.stride()
    return x.data_ptr(), row if one == 1 and row >= channels else _rows(x, what)[1]


def _conv_shape(x, weight, bias, n: int, silu):
    """(shape, taps, pointers of x, weight and bias, device) of a convolution's checked arguments."""
    code = _data(x, "x")
    if x.dim() != 2 or x.shape[1] < 1:
        raise ValueError(f"x must have shape (tokens, channels), got {tuple(x.shape)}")
    tokens, channels = x.shape
    dev = x.device
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2 or not 1 <= weight.shape[1] <= RN_CONV_MAX_TAPS:
        raise ValueError(f"weight must have shape (channels, taps) with 1..{RN_CONV_MAX_TAPS} taps")
    taps = weight.shape[1]
    _count(max(channels, n), "channels and n")
    xp, stride = _flat(x, "x", x.dtype, tokens, channels, dev)
    w, b = _like(weight, "weight", _F32, dev, (channels, taps)), _opt(bias, "bias", _F32, dev, (channels,))
    return rn_conv_shape(n, channels, taps, tokens, code, bool(silu), stride), taps, xp, w, b, dev


def causal_conv_step(x, weight, state, bias=None, stream_ids=None, silu: bool = True, out=None, stream=None):
    """One token for each of n streams, their windows updated in place (reuse_ops_causal_conv_step).

    x: [n][channels] float32 or bfloat16; weight: [channels][taps] float32,
    the last tap the token's own; state: [slots][taps - 1][channels] in x's
    dtype, the inputs before, oldest first; bias: [channels] float32 or None;
    stream_ids: [n] int32 distinct slots (None: 0..n-1).  Returns out
    [n][channels], which may be x.
    """
    if stream is not None:
        with _on(stream, x):
            return causal_conv_step(x, weight, state, bias, stream_ids, silu, out)
    _no_grad(x, weight, state, bias)
    n = x.shape[0] if isinstance(x, torch.Tensor) and x.dim() else 0
    shape, taps, xp, w, b, dev = _conv_shape(x, weight, bias, n, silu)
    slots = state.shape[0] if isinstance(state, torch.Tensor) and state.dim() else 0
    sp = _like(state, "state", x.dtype, dev, (_count(slots, "slots"), taps - 1, x.shape[1]))
    ids = _opt(stream_ids, "stream_ids", _I32, dev, (n,))
    if ids is None and slots < n:
        raise ValueError(f"{n} streams need as many slots, state has {slots}")
    if out is None:
        out = _empty(x)
    op = _like(out, "out", x.dtype, dev, x.shape)
    _launch(dev, load_ops().reuse_ops_causal_conv_step, ctypes.byref(shape), xp, w, b, ids, slots, sp, op)
    return out


def causal_conv(x, weight, bias=None, seq_off=None, n=None, state=None, final=None, silu: bool = True, out=None,
                stream=None):
    """All tokens of n sequences (reuse_ops_causal_conv).

    x: [tokens][channels], weight: [channels][taps], bias: [channels] or None,
    as for causal_conv_step; seq_off or n as for delta_forward, but tokens behind
    seq_off[n] are no sequence's: their results are left as they were.  state:
    [n][taps - 1][channels] in x's dtype, the inputs before each sequence
    (None: zeros); final: where the last ones go (made here if None; not
    state).  Returns (out, final).
    """
    if stream is not None:
        with _on(stream, x):
            return causal_conv(x, weight, bias, seq_off, n, state, final, silu, out)
    _no_grad(x, weight, bias, state)
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x must be a tensor of shape (tokens, channels)")
    n, off = _sequences(seq_off, n, x.shape[0], x.device)
    shape, taps, xp, w, b, dev = _conv_shape(x, weight, bias, n, silu)
    dims = (n, taps - 1, x.shape[1])
    sp = _opt(state, "state", x.dtype, dev, dims)
    if final is None:
        final = _empty(x, dims, x.dtype)
    fp = _like(final, "final", x.dtype, dev, dims)
    if out is None:
        out = _empty(x)
    op = _like(out, "out", x.dtype, dev, x.shape)
    _launch(dev, load_ops().reuse_ops_causal_conv, ctypes.byref(shape), xp, w, b, off, sp, fp, op)
    return out, final


def causal_conv_backward(dout, x, weight, bias=None, seq_off=None, n=None, state=None, dfinal=None, silu: bool = True,
                         want_dstate: bool = True, stream=None):
    """Gradients (dx, dweight, dbias, dstate) of causal_conv (reuse_ops_causal_conv_backward).

    The inputs are the forward call's; dout: dJ/dout, dfinal: dJ/dfinal in x's
    dtype or None.  dstate is None without want_dstate.
    """
    if stream is not None:
        with _on(stream, x):
            return causal_conv_backward(dout, x, weight, bias, seq_off, n, state, dfinal, silu, want_dstate)
    _no_grad(dout, x, weight, bias, state, dfinal)
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x must be a tensor of shape (tokens, channels)")
    n, off = _sequences(seq_off, n, x.shape[0], x.device)
    shape, taps, xp, w, b, dev = _conv_shape(x, weight, bias, n, silu)
    dims = (n, taps - 1, x.shape[1])
    sp = _opt(state, "state", x.dtype, dev, dims)
    do = _like(dout, "dout", x.dtype, dev, x.shape)
    df = _opt(dfinal, "dfinal", x.dtype, dev, dims)
    L = load_ops()
    need = L.reuse_ops_causal_conv_backward_scratch_bytes(ctypes.byref(shape))
    dx, dw, db = _empty(x), _empty(weight), _empty(x, x.shape[1], _F32)
    dstate = _empty(x, dims, x.dtype) if want_dstate else None
    scratch = _empty(x, need, torch.uint8)
    _launch(dev, L.reuse_ops_causal_conv_backward, ctypes.byref(shape), xp, w, b, off, sp, do, df, dx.data_ptr(),
            dw.data_ptr(), db.data_ptr(), None if dstate is None else dstate.data_ptr(), scratch.data_ptr(), need)
    return dx, dw, db, dstate


# ------------------------------------------------------------------ selective scan

def _scan_shape(u, dt, a, b, c, d, z, dt_bias, softplus, n: int):
    """(shape, inputs, channels, states, device) of a scan's checked arguments."""
    code = _data(u, "u")
    if u.dim() != 2 or u.shape[1] < 1:
        raise ValueError(f"u must have shape (tokens, channels), got {tuple(u.shape)}")
    tokens, channels = u.shape
    dev, dtype = u.device, u.dtype
    up, us = _flat(u, "u", dtype, tokens, channels, dev)
    dtp, dts = _flat(dt, "dt", dtype, tokens, channels, dev)
    zp, zs = (None, 0) if z is None else _flat(z, "z", dtype, tokens, channels, dev)
    groups, states, bs = _tokens(b, "b", dtype, tokens, dev)
    if channels % groups:
        raise ValueError(f"{channels} channels cannot share {groups} groups")
    groups_c, states_c, cs = _tokens(c, "c", dtype, tokens, dev)
    if groups_c != groups or states_c != states:
        raise ValueError("c must have b's shape")
    _count(max(channels, states, n), "channels, states and n")
    inputs = rn_scan_inputs(up, dtp, b.data_ptr(), c.data_ptr(), _like(a, "a", _F32, dev, (channels, states)),
                            _opt(d, "d", _F32, dev, (channels,)), zp, _opt(dt_bias, "dt_bias", _F32, dev, (channels,)))
    return (rn_scan_shape(n, channels, groups, states, tokens, code, bool(softplus), us, dts, bs, cs, zs), inputs,
            channels, states, dev)


def scan_step(u, dt, a, b, c, state, d=None, z=None, dt_bias=None, softplus: bool = True, stream_ids=None, out=None,
              stream=None):
    """One token for each of n streams, their states updated in place (reuse_ops_scan_step).

    u, dt, z: [n][channels], b, c: [n][groups][states] float32 or bfloat16; a:
    [channels][states], d, dt_bias: [channels] float32; d, z and dt_bias may be
    None.  state: [slots][channels][states] float32; stream_ids: [n] int32
    distinct slots (None: 0..n-1).  Returns out [n][channels], which may be u.
    """
    if stream is not None:
        with _on(stream, u):
            return scan_step(u, dt, a, b, c, state, d, z, dt_bias, softplus, stream_ids, out)
    _no_grad(u, dt, a, b, c, state, d, z, dt_bias)
    n = u.shape[0] if isinstance(u, torch.Tensor) and u.dim() else 0
    shape, inputs, channels, states, dev = _scan_shape(u, dt, a, b, c, d, z, dt_bias, softplus, n)
    slots = state.shape[0] if isinstance(state, torch.Tensor) and state.dim() else 0
    sp = _like(state, "state", _F32, dev, (_count(slots, "slots"), channels, states))
    ids = _opt(stream_ids, "stream_ids", _I32, dev, (n,))
    if ids is None and slots < n:
        raise ValueError(f"{n} streams need as many slots, state has {slots}")
    if out is None:
        out = _empty(u)
    op = _like(out, "out", u.dtype, dev, u.shape)
    _launch(dev, load_ops().reuse_ops_scan_step, ctypes.byref(shape), ctypes.byref(inputs), ids, slots, sp, op)
    return out


def _scan_supported(need: int, shape) -> int:
    if need == 0:                                  # re-run the call's own checks to report why
        _check(load_ops().reuse_ops_scan_step(ctypes.byref(shape), None, None, 0, None, None, None))
    return need


def scan_forward(u, dt, a, b, c, d=None, z=None, dt_bias=None, softplus: bool = True, seq_off=None, n=None, state=None,
                 final=None, save: bool = False, out=None, stream=None):
    """All tokens of n sequences (reuse_ops_scan_forward).

    The inputs as for scan_step, over tokens; seq_off or n as for
    causal_conv.  state: [n][channels][states] float32 before each sequence
    (None: zeros); final: where the last ones go (made here if None; it may be
    state).  Returns (out, final), with save also the buffer that scan_backward
    reads.
    """
    if stream is not None:
        with _on(stream, u):
            return scan_forward(u, dt, a, b, c, d, z, dt_bias, softplus, seq_off, n, state, final, save, out)
    _no_grad(u, dt, a, b, c, d, z, dt_bias, state)
    if not isinstance(u, torch.Tensor) or u.dim() != 2:
        raise ValueError("u must be a tensor of shape (tokens, channels)")
    n, off = _sequences(seq_off, n, u.shape[0], u.device)
    shape, inputs, channels, states, dev = _scan_shape(u, dt, a, b, c, d, z, dt_bias, softplus, n)
    dims = (n, channels, states)
    sp = _opt(state, "state", _F32, dev, dims)
    L = load_ops()
    need = _scan_supported(L.reuse_ops_scan_scratch_bytes(ctypes.byref(shape)), shape)
    if final is None:
        final = _empty(u, dims, _F32)
    fp = _like(final, "final", _F32, dev, dims)
    if out is None:
        out = _empty(u)
    op = _like(out, "out", u.dtype, dev, u.shape)
    scratch = _empty(u, need, torch.uint8)
    saved, kept, size = None, None, 0
    if save:
        size = L.reuse_ops_scan_saved_bytes(ctypes.byref(shape))
        saved = _empty(u, size, torch.uint8)
        kept = saved.data_ptr()
    _launch(dev, L.reuse_ops_scan_forward, ctypes.byref(shape), ctypes.byref(inputs), off, sp, fp, op, kept, size,
            scratch.data_ptr(), need)
    return (out, final, saved) if save else (out, final)


def scan_backward(dout, u, dt, a, b, c, d=None, z=None, dt_bias=None, softplus: bool = True, seq_off=None, n=None,
                  saved=None, dfinal=None, want_dstate: bool = True, stream=None):
    """Gradients (du, ddt, da, db, dc, dd, dz, ddt_bias, dstate) of scan_forward (reuse_ops_scan_backward).

    The inputs are the forward call's, saved its buffer; dout: dJ/dout, dfinal:
    dJ/dfinal or None.  dd, dz and ddt_bias are None where d, z and dt_bias
    are, dstate without want_dstate.
    """
    if stream is not None:
        with _on(stream, u):
            return scan_backward(dout, u, dt, a, b, c, d, z, dt_bias, softplus, seq_off, n, saved, dfinal, want_dstate)
    _no_grad(dout, u, dt, a, b, c, d, z, dt_bias, dfinal)
    if not isinstance(u, torch.Tensor) or u.dim() != 2:
        raise ValueError("u must be a tensor of shape (tokens, channels)")
    n, off = _sequences(seq_off, n, u.shape[0], u.device)
    shape, inputs, channels, states, dev = _scan_shape(u, dt, a, b, c, d, z, dt_bias, softplus, n)
    dims = (n, channels, states)
    do = _like(dout, "dout", u.dtype, dev, u.shape)
    df = _opt(dfinal, "dfinal", _F32, dev, dims)
    L = load_ops()
    need = _scan_supported(L.reuse_ops_scan_backward_scratch_bytes(ctypes.byref(shape)), shape)
    if not isinstance(saved, torch.Tensor):
        raise TypeError("saved must be the buffer of scan_forward(..., save=True)")
    sp = _like(saved, "saved", torch.uint8, dev, (L.reuse_ops_scan_saved_bytes(ctypes.byref(shape)),))
    du, ddt, da, db, dc = _empty(u), _empty(u), _empty(a), _empty(b), _empty(c)
    dd, dz, dbias = (None if t is None else _empty(t) for t in (d, z, dt_bias))
    dstate = _empty(u, dims, _F32) if want_dstate else None
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    grads = rn_scan_grads(*map(ptr, (du, ddt, db, dc, dz, da, dd, dbias, dstate)))
    scratch = _empty(u, need, torch.uint8)
    _launch(dev, L.reuse_ops_scan_backward, ctypes.byref(shape), ctypes.byref(inputs), off, sp, saved.numel(), do, df,
            ctypes.byref(grads), scratch.data_ptr(), need)
    return du, ddt, da, db, dc, dd, dz, dbias, dstate
