"""The feed-forward block of a language model: layer norm, gated feed-forward layer, dropout (gn.h, "THE FEED-FORWARD BLOCK").

    out = x + dropout(gated_ffn(layer_norm(x)))

Matrices are 2-D CUDA tensors of float32, bfloat16 or float16 with unit stride inside a row (rows may be apart, as in a view
of a wider matrix); all tensors of a call are on one device and, where not said otherwise, of one type.  A call enqueues on `stream`
(default: the current stream of that device), never synchronises, and returns new tensors that belong to that stream; it can be
captured into a CUDA graph once a call of its kind has run on the device.  Nothing here takes part in autograd: the backward
passes are calls of their own.  Bad arguments raise TypeError or ValueError, the library's own refusals GnError.
"""
from __future__ import annotations

import contextlib
import ctypes as C

import torch

from .binding import GnError, lib

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTIVATIONS = {"sigmoid": 0, "silu": 1, "gelu": 2, "gelu_tanh": 3, "relu": 4}


def _matrix(t, what, rows, cols, like):
    """(pointer, leading dimension) of a matrix argument."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: expected a CUDA tensor")
    if t.dtype != like.dtype or t.device != like.device:
        raise TypeError(f"{what}: expected a {like.dtype} tensor on {like.device}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        raise ValueError(f"{what}: expected shape ({rows}, {cols}), got {tuple(t.shape)}")
    ld, inner = t.stride()
    if cols > 1 and inner != 1:
        raise ValueError(f"{what}: expected unit stride inside a row")
    if rows > 1 and ld < cols:
        raise ValueError(f"{what}: its rows overlap")
    return t.data_ptr(), ld if rows > 1 else max(ld, cols)


def _vector(t, what, n, like, types):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != like.device or t.dtype not in types:
        raise TypeError(f"{what}: expected a tensor of {' or '.join(str(d) for d in types)} on {like.device}")
    if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{what}: expected {n} consecutive elements")
    return t.data_ptr()


def _first(t, what):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what}: expected a CUDA tensor")
    if t.dtype not in _TYPES:
        raise TypeError(f"{what}: expected float32, bfloat16 or float16, got {t.dtype}")
    if t.dim() != 2 or t.shape[1] < 1:
        raise ValueError(f"{what}: expected a matrix with at least one column, got shape {tuple(t.shape)}")
    return _TYPES[t.dtype]


@contextlib.contextmanager
def _elsewhere(device, stream):
    with torch.cuda.device(device), torch.cuda.stream(stream):
        yield stream.cuda_stream


def _on(t, stream):
    """Context in which allocations and launches go to the call's device and stream; gives the stream's handle."""
    if stream is None:
        if t.device.index == torch.cuda.current_device():
            return contextlib.nullcontext(torch.cuda.current_stream().cuda_stream)
        stream = torch.cuda.current_stream(t.device)
    elif stream.device != t.device:
        raise ValueError(f"the stream is one of {stream.device}, the tensors are on {t.device}")
    return _elsewhere(t.device, stream)


def _checked(status, err):
    if status != 0:
        raise GnError(status, err.value.decode())


def layer_norm(x, weight=None, bias=None, eps=1e-5, save=False, stream=None):
    """y = (x - mean) rstd weight + bias, row by row; with `save` (y, mean, rstd), the statistics in float32.

    weight, bias: [cols], each optional, both of x's type or both float32.
    """
    kind = _first(x, "x")
    rows, cols = x.shape
    px, ldx = _matrix(x, "x", rows, cols, x)
    wtype = next((t.dtype for t in (weight, bias) if isinstance(t, torch.Tensor)), x.dtype)
    if wtype not in (x.dtype, torch.float32):
        raise TypeError(f"weight and bias: expected {x.dtype} or float32, got {wtype}")
    pw, pb = _vector(weight, "weight", cols, x, (wtype,)), _vector(bias, "bias", cols, x, (wtype,))
    with _on(x, stream) as st:
        y = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        stats = torch.empty((2, rows), dtype=torch.float32, device=x.device) if save else None
        pm = stats.data_ptr() if save else None
        err = C.create_string_buffer(160)
        _checked(lib().gn_layer_norm(kind, _TYPES[wtype], rows, cols, px, ldx, pw, pb, eps, y.data_ptr(), cols, pm,
                                     pm + 4 * rows if save else None, st, err, 160), err)
    return (y, stats[0], stats[1]) if save else y


def layer_norm_grad(dy, x, mean, rstd, weight=None, add=None, stream=None):
    """(dx, dweight, dbias) of layer_norm; dweight and dbias have the weight's type (x's where there is no weight).

    mean, rstd: what layer_norm(..., save=True) has returned.  add: a gradient of x's shape that is added to dx (the residual path).
    """
    kind = _first(x, "x")
    rows, cols = x.shape
    px, ldx = _matrix(x, "x", rows, cols, x)
    pdy, ld_dy = _matrix(dy, "dy", rows, cols, x)
    pa, ld_add = _matrix(add, "add", rows, cols, x) if add is not None else (None, 0)
    pm, pr = _vector(mean, "mean", rows, x, (torch.float32,)), _vector(rstd, "rstd", rows, x, (torch.float32,))
    pw = _vector(weight, "weight", cols, x, (x.dtype, torch.float32))
    if pm is None or pr is None:
        raise TypeError("mean and rstd: expected what layer_norm(..., save=True) has returned")
    wtype = x.dtype if weight is None else weight.dtype
    n = lib().gn_layer_norm_grad_workspace(rows, cols)
    with _on(x, stream) as st:
        dx = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        dw, db = torch.empty(cols, dtype=wtype, device=x.device), torch.empty(cols, dtype=wtype, device=x.device)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device=x.device)
        err = C.create_string_buffer(160)
        _checked(lib().gn_layer_norm_grad(kind, _TYPES[wtype], rows, cols, pdy, ld_dy, px, ldx, pm, pr, pw, pa, ld_add, dx.data_ptr(), cols,
                                          dw.data_ptr(), db.data_ptr(), ws.data_ptr(), n, st, err, 160), err)
    return dx, dw, db


def dropout(x, p, key, step=0, residual=None, device_step=None, stream=None):
    """x / (1 - p) where the generator keeps an element, 0 elsewhere, plus the residual.

    The mask is a function of the element's number in x, of `key` and of `step` (integers, taken modulo 2^64): the same numbers give the same
    mask, so the backward pass is dropout(dy, p, key, step).  device_step: an int64 CUDA tensor of one element that is added to
    step when the kernel runs, for steps captured into a graph.
    """
    kind = _first(x, "x")
    rows, cols = x.shape
    px, ldx = _matrix(x, "x", rows, cols, x)
    pr, ld_res = _matrix(residual, "residual", rows, cols, x) if residual is not None else (None, 0)
    ps = None
    if device_step is not None:
        if not isinstance(device_step, torch.Tensor) or device_step.device != x.device or device_step.dtype != torch.int64:
            raise TypeError(f"device_step: expected an int64 tensor on {x.device}")
        if device_step.numel() != 1:
            raise ValueError("device_step: expected one element")
        ps = device_step.data_ptr()
    with _on(x, stream) as st:
        y = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        err = C.create_string_buffer(160)
        _checked(lib().gn_dropout(kind, rows, cols, px, ldx, pr, ld_res, y.data_ptr(), cols, p, key & 0xFFFFFFFFFFFFFFFF,
                                  step & 0xFFFFFFFFFFFFFFFF, ps, st, err, 160), err)
    return y


_Args = C.c_int64 * 27          # gn_ffn: type and act, rows, cols and inner, then pointer and leading dimension of twelve matrices
_NONE = (0, 0)


def _ffn_call(fn, backward, x, act, kind, rows, cols, inner, mats, st):
    handle = lib()
    args = _Args(kind | act << 32, rows, cols | inner << 32, *[v for m in mats for v in m])
    n = handle.gn_gated_ffn_workspace(args, backward)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=x.device)
    err = C.create_string_buffer(160)
    _checked(fn(args, ws.data_ptr(), n, st, err, 160), err)


def _ffn_inputs(x, w_gate, w_up, w_down, act):
    kind = _first(x, "x")
    if act not in ACTIVATIONS:
        raise ValueError(f"act: expected one of {', '.join(ACTIVATIONS)}, got {act!r}")
    _first(w_gate, "w_gate")
    rows, cols = x.shape
    inner = w_gate.shape[0]
    if inner < 1:
        raise ValueError("w_gate: expected at least one row")
    mats = [_matrix(x, "x", rows, cols, x), _matrix(w_gate, "w_gate", inner, cols, x), _matrix(w_up, "w_up", inner, cols, x),
            _matrix(w_down, "w_down", cols, inner, x)]
    return kind, ACTIVATIONS[act], rows, cols, inner, mats


def gated_ffn(x, w_gate, w_up, w_down, act="silu", save=False, stream=None):
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T; with `save` (y, gate, up), the two projections for the backward pass.

    x [rows][cols], w_gate and w_up [inner][cols], w_down [cols][inner]; act: "sigmoid", "silu", "gelu", "gelu_tanh" or "relu".
    """
    kind, a, rows, cols, inner, mats = _ffn_inputs(x, w_gate, w_up, w_down, act)
    with _on(x, stream) as st:
        y = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        gate = torch.empty((rows, inner), dtype=x.dtype, device=x.device) if save else None
        up = torch.empty((rows, inner), dtype=x.dtype, device=x.device) if save else None
        mats += [(y.data_ptr(), cols), (gate.data_ptr(), inner) if save else _NONE, (up.data_ptr(), inner) if save else _NONE]
        mats += [_NONE] * 5
        _ffn_call(lib().gn_gated_ffn, 0, x, a, kind, rows, cols, inner, mats, st)
    return (y, gate, up) if save else y


def gated_ffn_grad(dy, x, gate, up, w_gate, w_up, w_down, act="silu", stream=None):
    """(dx, dw_gate, dw_up, dw_down) of gated_ffn; gate, up: what gated_ffn(..., save=True) has returned."""
    kind, a, rows, cols, inner, mats = _ffn_inputs(x, w_gate, w_up, w_down, act)
    mats += [_NONE, _matrix(gate, "gate", rows, inner, x), _matrix(up, "up", rows, inner, x), _matrix(dy, "dy", rows, cols, x)]
    with _on(x, stream) as st:
        dx = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        dwg = torch.empty((inner, cols), dtype=x.dtype, device=x.device)
        dwu = torch.empty((inner, cols), dtype=x.dtype, device=x.device)
        dwd = torch.empty((cols, inner), dtype=x.dtype, device=x.device)
        mats += [(dx.data_ptr(), cols), (dwg.data_ptr(), cols), (dwu.data_ptr(), cols), (dwd.data_ptr(), inner)]
        _ffn_call(lib().gn_gated_ffn_grad, 1, x, a, kind, rows, cols, inner, mats, st)
    return dx, dwg, dwu, dwd


def gated_ffn_status(device=None, stream=None):
    """Synchronises and raises GnError (GN_ETIMEOUT) if a bounded wait of a gated_ffn call's kernels has run out on the device since the
    last look; results since then are invalid."""
    with torch.cuda.device(device if stream is None else stream.device):
        st = stream if stream is not None else torch.cuda.current_stream()
        err = C.create_string_buffer(160)
        _checked(lib().gn_gated_ffn_status(st.cuda_stream, err, 160), err)
