"""The feed-forward block of a language model: layer norm, gated feed-forward layer, dropout (gn.h, "THE FEED-FORWARD BLOCK").

    out = x + dropout(gated_ffn(layer_norm(x)))

Matrices are 2-D CUDA tensors of float32, bfloat16 or float16 with unit stride inside a row (rows may be apart, as in a view
of a wider matrix); all tensors of a call are on one device and, where not said otherwise, of one type.  A call enqueues on `stream`
(default: the current stream of that device), never synchronises, and returns new tensors that belong to that stream; it can be
captured into a CUDA graph once a call of its kind has run on the device.  A given `stream` does not wait for the current one, which the
caller sees to (Stream.wait_stream), but the arguments' memory is kept until it is done with them, whether or not the caller drops
them.  Nothing here takes part in autograd: the backward passes are calls of their own.  Bad arguments raise TypeError or ValueError,
the library's own refusals GnError.
"""
from __future__ import annotations

import ctypes as C
import threading
from array import array

import torch

from .binding import GnError, lib

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_WIDE = 1 << 31                          # widths are 32-bit words of the library's calls, and what does not fit would be cut off on the way
ACTIVATIONS = {"sigmoid": 0, "silu": 1, "gelu": 2, "gelu_tanh": 3, "relu": 4}

# A small call is bound by what the host does for it, so the ordinary case (contiguous tensors on the current device and stream) takes few steps:
# checks that look at a tensor once, the stream's handle without an object around it, an error buffer for each thread.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_here = threading.local()


def _err():
    try:
        return _here.err
    except AttributeError:
        _here.err = C.create_string_buffer(200)
        return _here.err


def _matrix(t, what, rows, cols, dtype, dev):
    """(pointer, leading dimension) of a matrix argument."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a CUDA tensor")
    if t.dtype is not dtype or t.get_device() != dev:
        raise TypeError(f"{what}: expected a {dtype} tensor on cuda:{dev}, got {t.dtype} on {t.device}")
    if t.shape != (rows, cols):
        raise ValueError(f"{what}: expected shape ({rows}, {cols}), got {tuple(t.shape)}")
    if t.is_contiguous():
        return t.data_ptr(), cols
    ld, inner = t.stride()
    if cols > 1 and inner != 1:
        raise ValueError(f"{what}: expected unit stride inside a row")
    if rows > 1 and ld < cols:
        raise ValueError(f"{what}: its rows overlap")
    return t.data_ptr(), ld if rows > 1 else max(ld, cols)


def _vector(t, what, n, dev, *types):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.get_device() != dev or t.dtype not in types:
        raise TypeError(f"{what}: expected a tensor of {' or '.join(str(d) for d in types)} on cuda:{dev}")
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{what}: expected {n} consecutive elements")
    return t.data_ptr()


def _first(t, what):
    """(dtype, device index, rows, cols) of the matrix that the others have to go with."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a CUDA tensor")
    dev, dtype = t.get_device(), t.dtype
    if dev < 0:
        raise TypeError(f"{what}: expected a CUDA tensor")
    if dtype not in _TYPES:
        raise TypeError(f"{what}: expected float32, bfloat16 or float16, got {dtype}")
    shape = t.shape
    if len(shape) != 2 or shape[1] < 1:
        raise ValueError(f"{what}: expected a matrix with at least one column, got shape {tuple(shape)}")
    if shape[1] >= _WIDE:
        raise ValueError(f"{what}: expected fewer than 2^31 columns, got shape {tuple(shape)}")
    return dtype, dev, shape[0], shape[1]


_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _elsewhere(call, dev, stream, *args):
    """call(*args) where allocations and launches go to the given device and stream, for calls that are not on the current ones."""
    if stream is None:
        with torch.cuda.device(dev):
            return call(*args)
    if not isinstance(stream, torch.Stream):             # (torch.cuda.Stream is one)
        raise TypeError(f"stream: expected a torch.cuda.Stream, got {type(stream).__name__}")
    if stream.device.type != "cuda" or stream.device.index != dev:
        raise ValueError(f"the stream is one of {stream.device}, the tensors are on cuda:{dev}")
    with torch.cuda.device(dev), torch.cuda.stream(stream):
        out = call(*args)
    for t in args:                       # (memory of another stream's may be dropped, and handed out again, before this one has read it)
        if isinstance(t, torch.Tensor):
            t.record_stream(stream)
    return out


def _checked(status, err):
    if status != 0:
        raise GnError(status, err.value.decode())


def layer_norm(x, weight=None, bias=None, eps=1e-5, save=False, stream=None):
    """y = (x - mean) rstd weight + bias, row by row; with `save` (y, mean, rstd), the statistics in float32.

    weight, bias: [cols], each optional, both of x's type or both float32.
    """
    dtype, dev, rows, cols = _first(x, "x")
    if stream is not None or dev != _device():
        return _elsewhere(layer_norm, dev, stream, x, weight, bias, eps, save)
    px, ldx = _matrix(x, "x", rows, cols, dtype, dev)
    wtype = dtype
    if isinstance(weight, torch.Tensor):
        wtype = weight.dtype
    elif isinstance(bias, torch.Tensor):
        wtype = bias.dtype
    if wtype is not dtype and wtype is not torch.float32:
        raise TypeError(f"weight and bias: expected {dtype} or float32, got {wtype}")
    pw, pb = _vector(weight, "weight", cols, dev, wtype), _vector(bias, "bias", cols, dev, wtype)
    y = x.new_empty(rows, cols)
    mean = rstd = pm = pr = None
    if save:
        mean, rstd = x.new_empty(rows, dtype=torch.float32), x.new_empty(rows, dtype=torch.float32)
        pm, pr = mean.data_ptr(), rstd.data_ptr()
    err = _err()
    status = lib().gn_layer_norm(_TYPES[dtype], _TYPES[wtype], rows, cols, px, ldx, pw, pb, float(eps), y.data_ptr(), cols, pm, pr, _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)
    return (y, mean, rstd) if save else y


def layer_norm_grad(dy, x, mean, rstd, weight=None, add=None, stream=None):
    """(dx, dweight, dbias) of layer_norm; dweight and dbias have the weight's type (x's where there is no weight).

    mean, rstd: what layer_norm(..., save=True) has returned.  add: a gradient of x's shape that is added to dx (the residual path).
    """
    dtype, dev, rows, cols = _first(x, "x")
    if stream is not None or dev != _device():
        return _elsewhere(layer_norm_grad, dev, stream, dy, x, mean, rstd, weight, add)
    px, ldx = _matrix(x, "x", rows, cols, dtype, dev)
    pdy, ld_dy = _matrix(dy, "dy", rows, cols, dtype, dev)
    pa, ld_add = _matrix(add, "add", rows, cols, dtype, dev) if add is not None else (None, 0)
    if mean is None or rstd is None:
        raise TypeError("mean and rstd: expected what layer_norm(..., save=True) has returned")
    pm, pr = _vector(mean, "mean", rows, dev, torch.float32), _vector(rstd, "rstd", rows, dev, torch.float32)
    pw = _vector(weight, "weight", cols, dev, dtype, torch.float32)
    wtype = dtype if weight is None else weight.dtype
    handle = lib()
    n = handle.gn_layer_norm_grad_workspace(rows, cols)              # (negative for sizes that the call is to refuse)
    dx, ws = x.new_empty(rows, cols), x.new_empty(max(n, 16) // x.element_size())
    if wtype is dtype:
        dw, db = x.new_empty(cols), x.new_empty(cols)
    else:
        dw, db = x.new_empty(cols, dtype=wtype), x.new_empty(cols, dtype=wtype)
    err = _err()
    status = handle.gn_layer_norm_grad(_TYPES[dtype], _TYPES[wtype], rows, cols, pdy, ld_dy, px, ldx, pm, pr, pw, pa, ld_add, dx.data_ptr(), cols,
                                       dw.data_ptr(), db.data_ptr(), ws.data_ptr(), n, _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)
    return dx, dw, db


def dropout(x, p, key, step=0, residual=None, device_step=None, stream=None):
    """x / (1 - p) where the generator keeps an element, 0 elsewhere, plus the residual.

    The mask is a function of the element's number in x, of `key` and of `step` (integers, taken modulo 2^64): the same numbers give the same
    mask, so the backward pass is dropout(dy, p, key, step).  device_step: an int64 CUDA tensor of one element that is added to
    step when the kernel runs, for steps captured into a graph.
    """
    dtype, dev, rows, cols = _first(x, "x")
    if stream is not None or dev != _device():
        return _elsewhere(dropout, dev, stream, x, p, key, step, residual, device_step)
    px, ldx = _matrix(x, "x", rows, cols, dtype, dev)
    pr, ld_res = _matrix(residual, "residual", rows, cols, dtype, dev) if residual is not None else (None, 0)
    ps = None
    if device_step is not None:
        if not isinstance(device_step, torch.Tensor) or device_step.get_device() != dev or device_step.dtype is not torch.int64:
            raise TypeError(f"device_step: expected an int64 tensor on cuda:{dev}")
        if device_step.numel() != 1:
            raise ValueError("device_step: expected one element")
        ps = device_step.data_ptr()
    y = x.new_empty(rows, cols)
    err = _err()
    status = lib().gn_dropout(_TYPES[dtype], rows, cols, px, ldx, pr, ld_res, y.data_ptr(), cols, float(p), key & 0xFFFFFFFFFFFFFFFF,
                              step & 0xFFFFFFFFFFFFFFFF, ps, _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)
    return y


_REST = [(0,) * (24 - 2 * k) for k in range(13)]       # gn_ffn: the members behind the k-th of its twelve matrices


def _ffn_inputs(x, w_gate, w_up, w_down, act):
    dtype, dev, rows, cols = _first(x, "x")
    a = ACTIVATIONS.get(act)
    if a is None:
        raise ValueError(f"act: expected one of {', '.join(ACTIVATIONS)}, got {act!r}")
    if not isinstance(w_gate, torch.Tensor) or w_gate.dim() != 2 or w_gate.shape[0] < 1:
        raise (ValueError if isinstance(w_gate, torch.Tensor) else TypeError)("w_gate: expected a matrix with at least one row")
    inner = w_gate.shape[0]
    if inner >= _WIDE:
        raise ValueError(f"w_gate: expected fewer than 2^31 rows, got shape {tuple(w_gate.shape)}")
    words = [_TYPES[dtype] | a << 32, rows, cols | inner << 32, *_matrix(x, "x", rows, cols, dtype, dev),
             *_matrix(w_gate, "w_gate", inner, cols, dtype, dev), *_matrix(w_up, "w_up", inner, cols, dtype, dev),
             *_matrix(w_down, "w_down", cols, inner, dtype, dev)]
    return dtype, dev, rows, cols, inner, words


def _ffn_call(fn, backward, x, dev, words, mats):
    """gn_ffn as 27 words: type and act, rows, cols and inner, then pointer and leading dimension of twelve matrices."""
    words.extend(_REST[mats])
    args = array("q", words)
    at = args.buffer_info()[0]
    n = lib().gn_gated_ffn_workspace(at, backward)
    ws = x.new_empty(max(n, 16) // x.element_size())
    err = _err()
    status = fn(at, ws.data_ptr(), n, _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)


def gated_ffn(x, w_gate, w_up, w_down, act="silu", save=False, stream=None):
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T; with `save` (y, gate, up), the two projections for the backward pass.

    x [rows][cols], w_gate and w_up [inner][cols], w_down [cols][inner]; act: "sigmoid", "silu", "gelu", "gelu_tanh" or "relu".
    gate and up are views of wider buffers where their 16-bit rows would not start on 16 bytes otherwise.
    """
    dtype, dev, rows, cols, inner, words = _ffn_inputs(x, w_gate, w_up, w_down, act)
    if stream is not None or dev != _device():
        return _elsewhere(gated_ffn, dev, stream, x, w_gate, w_up, w_down, act, save)
    y = x.new_empty(rows, cols)
    words += (y.data_ptr(), cols)
    if not save:
        _ffn_call(lib().gn_gated_ffn, 0, x, dev, words, 5)
        return y
    if dtype is not torch.float32 and inner % 8:     # rows that start on 16 bytes: the backward pass reads them without a copy
        ld = (inner + 7) // 8 * 8
        gate, up = x.new_empty(rows, ld)[:, :inner], x.new_empty(rows, ld)[:, :inner]
    else:
        ld, gate, up = inner, x.new_empty(rows, inner), x.new_empty(rows, inner)
    words += (gate.data_ptr(), ld, up.data_ptr(), ld)
    _ffn_call(lib().gn_gated_ffn, 0, x, dev, words, 7)
    return y, gate, up


def gated_ffn_grad(dy, x, gate, up, w_gate, w_up, w_down, act="silu", stream=None):
    """(dx, dw_gate, dw_up, dw_down) of gated_ffn; gate, up: what gated_ffn(..., save=True) has returned."""
    dtype, dev, rows, cols, inner, words = _ffn_inputs(x, w_gate, w_up, w_down, act)
    if stream is not None or dev != _device():
        return _elsewhere(gated_ffn_grad, dev, stream, dy, x, gate, up, w_gate, w_up, w_down, act)
    words += (0, 0, *_matrix(gate, "gate", rows, inner, dtype, dev), *_matrix(up, "up", rows, inner, dtype, dev), *_matrix(dy, "dy", rows, cols, dtype, dev))
    dx = x.new_empty(rows, cols)
    dwg, dwu, dwd = x.new_empty(inner, cols), x.new_empty(inner, cols), x.new_empty(cols, inner)
    words += (dx.data_ptr(), cols, dwg.data_ptr(), cols, dwu.data_ptr(), cols, dwd.data_ptr(), inner)
    _ffn_call(lib().gn_gated_ffn_grad, 1, x, dev, words, 12)
    return dx, dwg, dwu, dwd


def gated_ffn_status(device=None, stream=None):
    """Synchronises and raises GnError (GN_ETIMEOUT) if a bounded wait of a gated_ffn call's kernels has run out on the device since the
    last look; results since then are invalid."""
    with torch.cuda.device(device if stream is None else stream.device):
        st = stream if stream is not None else torch.cuda.current_stream()
        err = _err()
        _checked(lib().gn_gated_ffn_status(st.cuda_stream, err, 200), err)
