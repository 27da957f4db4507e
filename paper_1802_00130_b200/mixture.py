"""A mixture of experts in the place of a feed-forward layer (gn.h, "A MIXTURE OF EXPERTS").

    index, weight = route(logits, k)
    y = experts(x, index, weight, w_gate, w_up, w_down)        # sum over a token's experts of weight * ffn_expert(x)

What the feed-forward block's calls say of tensors, streams, graphs, errors and autograd holds here too: matrices are CUDA tensors of
float32, bfloat16 or float16 with unit stride inside a row, results are new tensors of the call's stream, backward passes are calls of their own.
"""
from __future__ import annotations

import struct
from array import array
from numbers import Real

import torch

from .binding import lib
from .feedforward import _TYPES, ACTIVATIONS, _checked, _device, _elsewhere, _err, _first, _matrix, _raw_stream, _vector

SCORES = {"softmax": 0, "sigmoid": 1}
_ONE = 0x3FF0000000000000                # 1.0 as a 64-bit word


def _score(score):
    s = SCORES.get(score)
    if s is None:
        raise ValueError(f"score: expected one of {', '.join(SCORES)}, got {score!r}")
    return s


def _table(t, what, rows, k, dtype, dev):
    """Pointer of a [rows][k] table of consecutive words."""
    if not isinstance(t, torch.Tensor) or t.get_device() != dev or t.dtype is not dtype:
        raise TypeError(f"{what}: expected a {dtype} tensor on cuda:{dev}")
    if t.shape != (rows, k) or not t.is_contiguous():
        raise ValueError(f"{what}: expected shape ({rows}, {k}), contiguous, got {tuple(t.shape)}")
    return t.data_ptr()


def _choices(index, tokens):
    """How many experts a token has in an index table."""
    if not isinstance(index, torch.Tensor):
        raise TypeError("index: expected a CUDA tensor")
    if index.dim() != 2 or index.shape[0] != tokens or index.shape[1] < 1:
        raise ValueError(f"index: expected shape ({tokens}, k), got {tuple(index.shape)}")
    return index.shape[1]


def _bits(scale):
    """A float as a 64-bit word."""
    if type(scale) is float and scale == 1.0:
        return _ONE
    if isinstance(scale, bool) or not isinstance(scale, Real):
        raise TypeError(f"scale: expected a number, got {type(scale).__name__}")
    if abs(scale) > 1e300:
        scale = float("inf")         # (which the library refuses; a whole number may be too large for a float)
    return struct.unpack("q", struct.pack("d", scale))[0]


def _whole(value, what):
    """A count, small enough for the library's 32-bit words."""
    if isinstance(value, bool) or not isinstance(value, int):
        raise TypeError(f"{what}: expected an int, got {type(value).__name__}")
    return max(-1, min(value, 0x7FFFFFFF))


def route(logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_best=1, renormalise=False, scale=1.0, stream=None):
    """(index, weight): the k experts of each row of logits [tokens][experts], the best first, int32, and their weights, float32.

    score: "softmax" or "sigmoid" of the logits.  bias: float32 [experts], added to the scores for the choice alone (balance); without one, experts are
    compared by their logits.  groups: neighbouring experts form so many groups, of which the top_groups with the largest sum of their
    group_best (1 or 2) best values remain.  Equal values go by the lower number, and no rounding decides an order.
    weight: the scores of the chosen, divided by their sum with `renormalise` (however small they are), times `scale`.  Logits of -inf have the score 0; a token that has
    chosen nothing else (or, with sigmoid, nothing above -700) has weights of 0.
    """
    dtype, dev, tokens, n = _first(logits, "logits")
    if stream is not None or dev != _device():
        return _elsewhere(route, dev, stream, logits, k, score, bias, groups, top_groups, group_best, renormalise, scale)
    kind = _score(score)
    if type(k) is not int or not 1 <= k <= n:
        _whole(k, "k")
        raise ValueError(f"k: expected 1 to {n}, got {k}")
    if not groups == top_groups == group_best == 1:
        groups, top_groups, group_best = _whole(groups, "groups"), _whole(top_groups, "top_groups"), _whole(group_best, "group_best")
    index, weight = logits.new_empty(tokens, k, dtype=torch.int32), logits.new_empty(tokens, k, dtype=torch.float32)
    args = array("q", (_TYPES[dtype] | kind << 32, tokens, n | k << 32, groups & 0xFFFFFFFF | top_groups << 32, group_best & 0xFFFFFFFF | (1 << 32 if renormalise else 0),
                       _bits(scale), *_matrix(logits, "logits", tokens, n, dtype, dev), _vector(bias, "bias", n, dev, torch.float32) or 0, index.data_ptr(),
                       weight.data_ptr(), 0, 0))
    err = _err()
    status = lib().gn_route(args.buffer_info()[0], _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)
    return index, weight


def route_grad(dweight, logits, index, score="softmax", renormalise=False, scale=1.0, stream=None):
    """dlogits of route, of the logits' type; dweight [tokens][k] float32, index: what route has returned (entries that are no expert take no part)."""
    dtype, dev, tokens, n = _first(logits, "logits")
    if stream is not None or dev != _device():
        return _elsewhere(route_grad, dev, stream, dweight, logits, index, score, renormalise, scale)
    k = _choices(index, tokens)
    if k >= 1 << 31:
        raise ValueError("index: expected a size below 2^31")
    kind = _score(score)
    dlogits = logits.new_empty(tokens, n)
    args = array("q", (_TYPES[dtype] | kind << 32, tokens, n | k << 32, 0, 1 << 32 if renormalise else 0, _bits(scale), *_matrix(logits, "logits", tokens, n, dtype, dev), 0,
                       _table(index, "index", tokens, k, torch.int32, dev), _table(dweight, "dweight", tokens, k, torch.float32, dev), dlogits.data_ptr(), n))
    err = _err()
    status = lib().gn_route_grad(args.buffer_info()[0], _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)
    return dlogits


def _stack(t, what, experts, rows, cols, dtype, dev):
    """(pointer, leading dimension, stride) of a matrix of every expert."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a CUDA tensor")
    if t.dtype is not dtype or t.get_device() != dev:
        raise TypeError(f"{what}: expected a {dtype} tensor on cuda:{dev}, got {t.dtype} on {t.device}")
    if t.shape != (experts, rows, cols):
        raise ValueError(f"{what}: expected shape ({experts}, {rows}, {cols}), got {tuple(t.shape)}")
    if t.is_contiguous():
        return t.data_ptr(), cols, rows * cols
    stride, ld, inner = t.stride()
    if cols > 1 and inner != 1:
        raise ValueError(f"{what}: expected unit stride inside a row")
    if rows == 1:
        ld = max(ld, cols)
    if ld < cols:
        raise ValueError(f"{what}: its rows overlap")
    if experts == 1:
        stride = max(stride, rows * ld)
    if stride < (rows - 1) * ld + cols:
        raise ValueError(f"{what}: its experts overlap")
    return t.data_ptr(), ld, stride


_NONE2, _NONE3 = (0, 0), (0, 0, 0)


def _mixture(x, index, weight, w_gate, w_up, w_down, act):
    """(type, device, sizes, first words of a gn_mixture, the three weights' words)."""
    dtype, dev, tokens, cols = _first(x, "x")
    a = ACTIVATIONS.get(act)
    if a is None:
        raise ValueError(f"act: expected one of {', '.join(ACTIVATIONS)}, got {act!r}")
    if not isinstance(w_gate, torch.Tensor):
        raise TypeError("w_gate: expected a CUDA tensor")
    if w_gate.dim() != 3 or w_gate.shape[0] < 1 or w_gate.shape[1] < 1:
        raise ValueError(f"w_gate: expected shape (experts, inner, {cols}), got {tuple(w_gate.shape)}")
    experts, inner = w_gate.shape[0], w_gate.shape[1]
    k = _choices(index, tokens)
    if max(cols, inner, experts, k) >= 1 << 31:
        raise ValueError("x, w_gate and index: expected sizes below 2^31")
    head = [_TYPES[dtype] | a << 32, tokens, cols | inner << 32, experts | k << 32, _table(index, "index", tokens, k, torch.int32, dev),
            _table(weight, "weight", tokens, k, torch.float32, dev)]
    stacks = (*_stack(w_gate, "w_gate", experts, inner, cols, dtype, dev), *_stack(w_up, "w_up", experts, inner, cols, dtype, dev),
              *_stack(w_down, "w_down", experts, cols, inner, dtype, dev))
    return dtype, dev, tokens, cols, inner, experts, k, head, stacks


def _mixture_call(fn, backward, x, dev, words):
    args = array("q", words)
    at = args.buffer_info()[0]
    n = lib().gn_experts_workspace(at, backward)
    ws = x.new_empty(max(n, 16) // x.element_size())
    err = _err()
    status = fn(at, ws.data_ptr(), n, _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)


def experts(x, index, weight, w_gate, w_up, w_down, act="silu", save=False, stream=None):
    """y = sum over a token's k experts of weight * (act(x w_gate^T) * (x w_up^T)) w_down^T; with `save` (y, gate, up), the projections for the backward pass.

    x [tokens][cols]; index (int32) and weight (float32) [tokens][k] as route gives them, an index that is no expert adds nothing; w_gate, w_up
    [experts][inner][cols], w_down [experts][cols][inner]; act as in gated_ffn.  gate and up: [tokens k][inner], row t k + j that of the token's j-th choice (not written
    where that is no expert); views of wider buffers where their 16-bit rows would not start on 16 bytes otherwise.
    """
    dtype, dev, tokens, cols, inner, n, k, head, stacks = _mixture(x, index, weight, w_gate, w_up, w_down, act)
    if stream is not None or dev != _device():
        return _elsewhere(experts, dev, stream, x, index, weight, w_gate, w_up, w_down, act, save)
    px = _matrix(x, "x", tokens, cols, dtype, dev)
    y = x.new_empty(tokens, cols)
    gate = up = None
    if save:
        ld = inner if dtype is torch.float32 else (inner + 7) // 8 * 8
        gate, up = (x.new_empty(tokens * k, ld)[:, :inner] for _ in range(2))
    saved = (gate.data_ptr(), ld, up.data_ptr(), ld) if save else (0, 0, 0, 0)
    _mixture_call(lib().gn_experts, 0, x, dev, (*head, 0, *px, y.data_ptr(), cols, *saved, *_NONE2, *_NONE2, *stacks, *_NONE3, *_NONE3, *_NONE3))
    return (y, gate, up) if save else y


def experts_grad(dy, x, index, weight, gate, up, w_gate, w_up, w_down, act="silu", stream=None):
    """(dx, dweight, dw_gate, dw_up, dw_down) of experts; gate, up: what experts(..., save=True) has returned.  dweight (float32): 0 where there is no expert."""
    dtype, dev, tokens, cols, inner, n, k, head, stacks = _mixture(x, index, weight, w_gate, w_up, w_down, act)
    if stream is not None or dev != _device():
        return _elsewhere(experts_grad, dev, stream, dy, x, index, weight, gate, up, w_gate, w_up, w_down, act)
    mats = (*_matrix(x, "x", tokens, cols, dtype, dev), *_NONE2, *_matrix(gate, "gate", tokens * k, inner, dtype, dev),
            *_matrix(up, "up", tokens * k, inner, dtype, dev), *_matrix(dy, "dy", tokens, cols, dtype, dev))
    dx, dweight = x.new_empty(tokens, cols), x.new_empty(tokens, k, dtype=torch.float32)
    dwg, dwu, dwd = x.new_empty(n, inner, cols), x.new_empty(n, inner, cols), x.new_empty(n, cols, inner)
    each = inner * cols
    _mixture_call(lib().gn_experts_grad, 1, x, dev, (*head, dweight.data_ptr(), *mats, dx.data_ptr(), cols, *stacks, dwg.data_ptr(), cols, each, dwu.data_ptr(), cols,
                                                     each, dwd.data_ptr(), inner, each))
    return dx, dweight, dwg, dwu, dwd
