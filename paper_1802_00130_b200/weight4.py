"""4-bit weights with a scale for each group of a row, and the products of a few tokens with them (gn.h, "4-BIT WEIGHTS").

    w = quantize4(weights)                 # or pack4(q, scale): laid out once
    y = matvec4(x, w)                      # x [tokens][cols], w [rows][cols]
    y = gated_ffn4(x, w_gate, w_up, w_down)
    y = gated_ffn4(x, w_gate, w_up, w_down, index=index, weight=weight)      # experts, as route has chosen them

Made for a decoder's few tokens: 32 at a time read and unpack all weights again.  A prompt goes through the unpacked weights in less time (from 160 tokens on for a layer of
4096 x 8192, from 2600 for 4 of 64 experts of 2048 x 1024),

    y = gated_ffn(x, *(unpack4(w) for w in (w_gate, w_up, w_down)))                # or experts(x, index, weight, ...)

What the feed-forward block's calls say of tensors, streams, graphs, errors and autograd holds here too.
"""
from __future__ import annotations

from array import array
from dataclasses import dataclass

import torch

from .binding import lib
from .mixture import _choices, _stack, _table, _whole
from .feedforward import _TYPES, ACTIVATIONS, _checked, _device, _elsewhere, _err, _first, _matrix, _raw_stream


@dataclass(frozen=True)
class Weight4:
    """4-bit weights of one matrix [rows][cols] (experts: None) or of every expert's, in the library's layout; made by pack4 and quantize4, or of what they have made (a
    copy on another device, a file)."""
    q: torch.Tensor
    scale: torch.Tensor
    experts: int | None
    rows: int
    cols: int
    group: int

    def __post_init__(self):
        """The products read as many bytes as the sizes say."""
        if not isinstance(self.q, torch.Tensor) or self.q.dtype is not torch.uint8 or not isinstance(self.scale, torch.Tensor) or self.scale.dtype not in _TYPES:
            raise TypeError("expected q as uint8 and scale as float32, bfloat16 or float16 tensors")
        n, rows, cols = 1 if self.experts is None else _whole(self.experts, "experts"), _whole(self.rows, "rows"), _whole(self.cols, "cols")
        bytes_, scales = lib().gn_weight4_bytes(n, rows, cols), lib().gn_weight4_scales(n, rows, cols, _whole(self.group, "group"))
        if scales < 0 or (self.q.numel(), self.scale.numel()) != (bytes_, scales) or not self.q.is_contiguous() or not self.scale.is_contiguous():
            raise ValueError(f"expected {bytes_} consecutive bytes and {scales} consecutive scales for {self.shape} in groups of {self.group}, "
                             f"got {self.q.numel()} and {self.scale.numel()}")

    @property
    def shape(self):
        return (self.rows, self.cols) if self.experts is None else (self.experts, self.rows, self.cols)

    @property
    def dtype(self):
        """That of the scales, and of the tokens that it goes with."""
        return self.scale.dtype

    @property
    def device(self):
        return self.q.device


def _flat(t, what):
    """(device, experts or None, rows, cols) of a matrix or of every expert's."""
    if not isinstance(t, torch.Tensor) or t.get_device() < 0:
        raise TypeError(f"{what}: expected a CUDA tensor")
    if t.dim() not in (2, 3) or 0 in t.shape:
        raise ValueError(f"{what}: expected shape (rows, cols) or (experts, rows, cols), got {tuple(t.shape)}")
    return (t.get_device(), t.shape[0] if t.dim() == 3 else None, *t.shape[-2:])


def _room(t, dtype, n, rows, cols, group):
    """Tensors for the layout."""
    if not isinstance(group, int) or group not in (32, 64, 128):
        raise ValueError(f"group: expected 32, 64 or 128, got {group!r}")
    bytes_, scales = lib().gn_weight4_bytes(_whole(n, "experts"), rows, cols), lib().gn_weight4_scales(_whole(n, "experts"), rows, cols, group)
    if bytes_ < 0:
        raise ValueError(f"expected up to 1024 experts of up to 2^20 rows and columns with fewer than 2^31 weights, got ({n}, {rows}, {cols})")
    return t.new_empty(bytes_, dtype=torch.uint8), t.new_empty(scales, dtype=dtype)


def pack4(q, scale, group=128, stream=None):
    """Weight4 of weights scale (q - 8): q uint8 [rows][cols] or [experts][rows][cols] with values of 0 to 15 (the low four bits count), scale [...][rows][groups] of the
    type that the tokens will have; `group` (32, 64 or 128) neighbouring columns share a scale, the last ones of a row may be fewer."""
    dev, experts, rows, cols = _flat(q, "q")
    if stream is not None or dev != _device():
        return _elsewhere(pack4, dev, stream, q, scale, group)
    if q.dtype is not torch.uint8:
        raise TypeError(f"q: expected uint8, got {q.dtype}")
    if not isinstance(scale, torch.Tensor) or scale.get_device() != dev or scale.dtype not in _TYPES:
        raise TypeError(f"scale: expected a tensor of float32, bfloat16 or float16 on cuda:{dev}")
    n = 1 if experts is None else experts
    to_q, to_scale = _room(q, scale.dtype, n, rows, cols, group)
    if scale.shape != (*q.shape[:-1], -(-cols // group)) or not scale.is_contiguous():
        raise ValueError(f"scale: expected shape {(*q.shape[:-1], -(-cols // group))}, contiguous, got {tuple(scale.shape)}")
    at = _stack(q if experts is not None else q[None], "q", n, rows, cols, torch.uint8, dev)
    err = _err()
    _checked(lib().gn_pack4(_TYPES[scale.dtype], n, rows, cols, group, *at, scale.data_ptr(), to_q.data_ptr(), to_scale.data_ptr(), _raw_stream(dev), err, 200), err)
    return Weight4(to_q, to_scale, experts, rows, cols, group)


def quantize4(w, group=128, stream=None):
    """Weight4 nearest to w [rows][cols] or [experts][rows][cols]: a group's scale is its largest magnitude / 7, rounded to w's type."""
    dev, experts, rows, cols = _flat(w, "w")
    if stream is not None or dev != _device():
        return _elsewhere(quantize4, dev, stream, w, group)
    if w.dtype not in _TYPES:
        raise TypeError(f"w: expected float32, bfloat16 or float16, got {w.dtype}")
    n = 1 if experts is None else experts
    q, scale = _room(w, w.dtype, n, rows, cols, group)
    at = _stack(w if experts is not None else w[None], "w", n, rows, cols, w.dtype, dev)
    err = _err()
    _checked(lib().gn_quantize4(_TYPES[w.dtype], n, rows, cols, group, *at, q.data_ptr(), scale.data_ptr(), _raw_stream(dev), err, 200), err)
    return Weight4(q, scale, experts, rows, cols, group)


def _weight4(w, what, dtype=None, dev=None):
    if not isinstance(w, Weight4):
        raise TypeError(f"{what}: expected a Weight4, got {type(w).__name__}")
    if dtype is None and not 0 <= w.q.get_device() == w.scale.get_device():
        raise TypeError(f"{what}: expected CUDA tensors of one device, got {w.q.device} and {w.scale.device}")
    if dtype is not None and (w.scale.dtype is not dtype or w.q.get_device() != dev or w.scale.get_device() != dev):
        raise TypeError(f"{what}: expected scales of {dtype} on cuda:{dev}, got {w.scale.dtype} on {w.device}")
    return w.q.data_ptr(), w.scale.data_ptr()


def unpack4(w, stream=None):
    """What 4-bit weights stand for, in their scales' type."""
    pq, ps = _weight4(w, "w")
    dev = w.q.get_device()
    if stream is not None or dev != _device():
        out = _elsewhere(unpack4, dev, stream, w)
        _used_on(stream, w)
        return out
    out, err = w.scale.new_empty(w.shape), _err()
    _checked(lib().gn_unpack4(_TYPES[w.dtype], w.experts or 1, w.rows, w.cols, w.group, pq, ps, out.data_ptr(), w.cols, w.rows * w.cols, _raw_stream(dev), err, 200), err)
    return out


def _used_on(stream, *weights):
    """Weights that a given stream reads are kept until it is done with them."""
    if stream is not None:
        for w in weights:
            w.q.record_stream(stream)
            w.scale.record_stream(stream)


def matvec4(x, w, stream=None):
    """y [tokens][rows] = x [tokens][cols] w^T, in x's type, which has to be that of the scales.  Made for few tokens (32 at a time)."""
    dtype, dev, tokens, cols = _first(x, "x")
    pq, ps = _weight4(w, "w", dtype, dev)
    if w.experts is not None or w.cols != cols:
        raise ValueError(f"w: expected shape (rows, {cols}), got {w.shape}")
    if stream is not None or dev != _device():
        out = _elsewhere(matvec4, dev, stream, x, w)
        _used_on(stream, w)
        return out
    px, ldx = _matrix(x, "x", tokens, cols, dtype, dev)
    y = x.new_empty(tokens, w.rows)
    ws, n = 0, 0
    if dtype is torch.float32 or cols & 7 or ldx & 7 or px & 15:
        n = (6 if dtype is torch.float32 else 2) * tokens * ((cols + 7) & ~7)      # (gn_matvec4_workspace's)
        room = x.new_empty(max(n, 16) // x.element_size())
        ws = room.data_ptr()
    err = _err()
    status = lib().gn_matvec4(_TYPES[dtype], tokens, w.rows, cols, w.group, px, ldx, pq, ps, y.data_ptr(), w.rows, ws, n, _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)
    return y


def gated_ffn4(x, w_gate, w_up, w_down, act="silu", index=None, weight=None, stream=None):
    """gated_ffn on 4-bit weights; with index (int32) and weight (float32), both [tokens][k] as route gives them, experts on 4-bit weights of every expert.

    w_gate, w_up: Weight4 of [inner][cols] ([experts][inner][cols]), w_down of [cols][inner]; one group size, scales of x's type.
    """
    dtype, dev, tokens, cols = _first(x, "x")
    a = ACTIVATIONS.get(act)
    if a is None:
        raise ValueError(f"act: expected one of {', '.join(ACTIVATIONS)}, got {act!r}")
    at = [_weight4(w, what, dtype, dev) for w, what in ((w_gate, "w_gate"), (w_up, "w_up"), (w_down, "w_down"))]
    n, inner = w_gate.experts, w_gate.rows
    for w, what, shape in ((w_gate, "w_gate", (inner, cols)), (w_up, "w_up", (inner, cols)), (w_down, "w_down", (cols, inner))):
        if w.experts != n or (w.rows, w.cols) != shape or w.group != w_gate.group:
            raise ValueError(f"{what}: expected shape {shape if n is None else (n, *shape)} in groups of {w_gate.group}, got {w.shape} in groups of {w.group}")
    if (index is None) != (n is None) or (index is None) != (weight is None):
        raise ValueError("index and weight: expected with weights of experts, and with those alone")
    if stream is not None or dev != _device():
        out = _elsewhere(gated_ffn4, dev, stream, x, w_gate, w_up, w_down, act, index, weight)
        _used_on(stream, w_gate, w_up, w_down)
        return out
    k, pi, pw = 1, 0, 0
    if index is not None:
        k = _choices(index, tokens)
        if k >= 1 << 31:
            raise ValueError("index: expected a size below 2^31")
        pi, pw = _table(index, "index", tokens, k, torch.int32, dev), _table(weight, "weight", tokens, k, torch.float32, dev)
    y = x.new_empty(tokens, cols)
    args = array("q", (_TYPES[dtype] | a << 32, tokens, cols | inner << 32, (n or 1) | k << 32, w_gate.group, pi, pw, *_matrix(x, "x", tokens, cols, dtype, dev),
                       y.data_ptr(), cols, *at[0], *at[1], *at[2]))
    p, handle = args.buffer_info()[0], lib()
    need = handle.gn_gated_ffn4_workspace(p)
    ws = x.new_empty(max(need, 16) // x.element_size() + 1)
    err = _err()
    status = handle.gn_gated_ffn4(p, ws.data_ptr(), need, _raw_stream(dev), err, 200)
    if status:
        _checked(status, err)
    return y
