"""A mixture of experts in the place of a feed-forward layer (gn.h, "A MIXTURE OF EXPERTS").

    index, weight = route(logits, k)
    y = experts(x, index, weight, w_gate, w_up, w_down)        # sum over a token's experts of weight * ffn_expert(x)

What the feed-forward block's calls say of tensors, streams, graphs, errors and autograd holds here too: matrices are CUDA tensors of
float32, bfloat16 or float16 with unit stride inside a row, results are new tensors of the call's stream, backward passes are calls of their own.
"""
from __future__ import annotations

import torch

from .binding import lib
from .feedforward import _TYPES, _checked, _device, _elsewhere, _err, _first, _matrix, _raw_stream, _vector

SCORES = {"softmax": 0, "sigmoid": 1}


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
    weight: the scores of the chosen, divided by their sum with `renormalise`, times `scale`.  Logits of -inf have the score 0.
    """
    dtype, dev, tokens, n = _first(logits, "logits")
    if stream is not None or dev != _device():
        return _elsewhere(route, dev, stream, logits, k, score, bias, groups, top_groups, group_best, renormalise, scale)
    pl, ld = _matrix(logits, "logits", tokens, n, dtype, dev)
    pb = _vector(bias, "bias", n, dev, torch.float32)
    kind, k = _score(score), _whole(k, "k")
    if not 1 <= k <= n:
        raise ValueError(f"k: expected 1 to {n}, got {k}")
    index, weight = logits.new_empty(tokens, k, dtype=torch.int32), logits.new_empty(tokens, k, dtype=torch.float32)
    err = _err()
    status = lib().gn_route(_TYPES[dtype], kind, tokens, n, k, pl, ld, pb, _whole(groups, "groups"), _whole(top_groups, "top_groups"),
                            _whole(group_best, "group_best"), 1 if renormalise else 0, float(scale), index.data_ptr(), weight.data_ptr(),
                            _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)
    return index, weight


def route_grad(dweight, logits, index, score="softmax", renormalise=False, scale=1.0, stream=None):
    """dlogits of route, of the logits' type; dweight [tokens][k] float32, index: what route has returned (entries that are no expert take no part)."""
    dtype, dev, tokens, n = _first(logits, "logits")
    if stream is not None or dev != _device():
        return _elsewhere(route_grad, dev, stream, dweight, logits, index, score, renormalise, scale)
    pl, ld = _matrix(logits, "logits", tokens, n, dtype, dev)
    k = _choices(index, tokens)
    pi, pw = _table(index, "index", tokens, k, torch.int32, dev), _table(dweight, "dweight", tokens, k, torch.float32, dev)
    kind = _score(score)
    dlogits = logits.new_empty(tokens, n)
    err = _err()
    status = lib().gn_route_grad(_TYPES[dtype], kind, tokens, n, k, pw, pl, ld, pi, 1 if renormalise else 0, float(scale), dlogits.data_ptr(), n,
                                 _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)
    return dlogits
