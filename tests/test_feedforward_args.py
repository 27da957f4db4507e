"""Refusals of the feed-forward block's calls: nothing is launched, so no device is needed."""
import ctypes as C

import pytest
import torch

import paper_1802_00130_b200 as gn

P = C.c_void_p(1 << 20)            # an aligned address that no refused call looks at


def refused(fn, *args):
    err = C.create_string_buffer(200)
    assert fn(*args, err, 200) == 1            # GN_EINVAL
    assert err.value
    return err.value.decode()


def norm(**change):
    a = dict(type=1, wtype=1, rows=4, cols=8, x=P, ldx=8, w=None, b=None, eps=1e-5, y=C.c_void_p(1 << 21), ldy=8, mean=None, rstd=None, st=None)
    a.update(change)
    return refused(gn.lib().gn_layer_norm, *a.values())


@pytest.mark.parametrize("change,word", [
    (dict(type=3), "type"), (dict(type=0, wtype=1), "weight's type"), (dict(type=1, wtype=2), "weight's type"), (dict(rows=-1), "rows"),
    (dict(rows=1 << 31), "rows"), (dict(cols=0), "cols"), (dict(cols=(1 << 20) + 1), "cols"), (dict(eps=-1e-9), "eps"),
    (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"), (dict(x=None), "x:"), (dict(ldx=7), "x:"), (dict(y=None), "y:"),
    (dict(ldy=7), "y:"), (dict(x=C.c_void_p((1 << 20) + 1)), "x:"), (dict(w=C.c_void_p(3)), "weight"), (dict(b=C.c_void_p(3)), "bias"),
    (dict(mean=C.c_void_p(6)), "mean"), (dict(y=P, ldy=16), "place of x")])
def test_layer_norm_refuses(change, word):
    assert word in norm(**change)


def norm_grad(**change):
    a = dict(type=1, wtype=0, rows=4, cols=8, dy=P, ld_dy=8, x=C.c_void_p(1 << 21), ldx=8, mean=P, rstd=P, w=None, add=None, ld_add=0,
             dx=C.c_void_p(1 << 22), ld_dx=8, dw=P, db=P, ws=P, n=1 << 30, st=None)
    a.update(change)
    return refused(gn.lib().gn_layer_norm_grad, *a.values())


@pytest.mark.parametrize("change,word", [
    (dict(type=-1), "type"), (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(dy=None), "dy"), (dict(ld_dy=7), "dy"), (dict(x=None), "x:"),
    (dict(mean=None), "mean"), (dict(rstd=None), "rstd"), (dict(add=P, ld_add=7), "add"), (dict(ld_dx=7), "dx"), (dict(dw=C.c_void_p(2)), "weight"),
    (dict(ws=None), "workspace"), (dict(ws=C.c_void_p(8)), "workspace"), (dict(n=8), "workspace"), (dict(dx=P, ld_dx=16), "place"),
    (dict(dx=C.c_void_p(1 << 21)), "place")])
def test_layer_norm_grad_refuses(change, word):
    assert word in norm_grad(**change)


def drop(**change):
    a = dict(type=1, rows=4, cols=8, x=P, ldx=8, res=None, ld_res=0, y=C.c_void_p(1 << 21), ldy=8, p=0.1, key=1, step=2, d_step=None, st=None)
    a.update(change)
    return refused(gn.lib().gn_dropout, *a.values())


@pytest.mark.parametrize("change,word", [
    (dict(type=7), "type"), (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(p=-0.1), "p must"), (dict(p=1.0000001), "p must"),
    (dict(p=float("nan")), "p must"), (dict(x=None), "x:"), (dict(ldx=7), "x:"), (dict(res=P, ld_res=7), "residual"), (dict(y=None), "y:"),
    (dict(d_step=C.c_void_p(4)), "d_step"), (dict(y=P, ldy=9), "place")])
def test_dropout_refuses(change, word):
    assert word in drop(**change)


def ffn_args(**change):
    """gn_ffn as 27 words: type and act, rows, cols and inner, then pointer and leading dimension of twelve matrices."""
    names = ["x", "w_gate", "w_up", "w_down", "y", "gate", "up", "dy", "dx", "dw_gate", "dw_up", "dw_down"]
    a = dict(type=1, act=1, rows=4, cols=8, inner=16)
    a.update({n: (1 << (20 + i), 16) for i, n in enumerate(names)})
    a.update(change)
    words = [a["type"] | a["act"] << 32, a["rows"], a["cols"] | a["inner"] << 32]
    return (C.c_int64 * 27)(*words, *[v for n in names for v in a[n]])


COMMON = [(dict(type=5), "type"), (dict(act=5), "act"), (dict(rows=-1), "rows"), (dict(cols=0), "cols"), (dict(inner=0), "cols"),
          (dict(cols=1 << 16, inner=1 << 15), "product"), (dict(x=(0, 16)), "x:"), (dict(x=(1 << 20, 7)), "x:"), (dict(w_gate=(0, 8)), "w_gate"),
          (dict(w_up=(1 << 20, 7)), "w_up"), (dict(w_down=(1 << 20, 15)), "w_down"), (dict(gate=(1 << 20, 15)), "gate"), (dict(up=(3, 16)), "up")]


@pytest.mark.parametrize("change,word", COMMON + [(dict(y=(0, 8)), "y:")])
def test_gated_ffn_refuses(change, word):
    args = ffn_args(**change)
    assert word in refused(gn.lib().gn_gated_ffn, args, P, 1 << 40, None)
    assert gn.lib().gn_gated_ffn_workspace(args, 0) < 0


@pytest.mark.parametrize("change,word", COMMON + [(dict(gate=(0, 16)), "gate"), (dict(up=(0, 16)), "up"), (dict(dy=(0, 8)), "dy"),
                                                  (dict(dx=(1 << 20, 7)), "dx"), (dict(dw_gate=(1 << 20, 7)), "dw_gate"),
                                                  (dict(dw_up=(1, 16)), "dw_up"), (dict(dw_down=(1 << 20, 15)), "dw_down")])
def test_gated_ffn_grad_refuses(change, word):
    args = ffn_args(**change)
    assert word in refused(gn.lib().gn_gated_ffn_grad, args, P, 1 << 40, None)
    assert gn.lib().gn_gated_ffn_workspace(args, 1) < 0


@pytest.mark.parametrize("fn", ["gn_gated_ffn", "gn_gated_ffn_grad"])
def test_gated_ffn_refuses_a_bad_workspace(fn):
    args = ffn_args()
    need = gn.lib().gn_gated_ffn_workspace(args, fn.endswith("grad"))
    assert need > 0
    for ws, n in ((None, need), (C.c_void_p((1 << 20) + 8), need), (P, need - 1)):
        assert "workspace" in refused(getattr(gn.lib(), fn), args, ws, n, None)
    assert "no arguments" in refused(getattr(gn.lib(), fn), None, P, need, None)


def test_no_error_buffer_is_fine():
    assert gn.lib().gn_dropout(9, 1, 1, P, 1, None, 0, P, 1, 0.1, 0, 0, None, None, None, 0) == 1
    assert gn.lib().gn_gated_ffn(None, P, 1, None, None, 0) == 1


def test_the_binding_refuses_tensors_that_are_not_on_a_device():
    x = torch.zeros(4, 8)
    for call in (lambda: gn.layer_norm(x), lambda: gn.layer_norm_grad(x, x, x[:, 0], x[:, 0]), lambda: gn.dropout(x, 0.1, 1),
                 lambda: gn.gated_ffn(x, x, x, x), lambda: gn.gated_ffn_grad(x, x, x, x, x, x, x)):
        with pytest.raises(TypeError, match="CUDA"):
            call()


class OnDevice(torch.Tensor):
    """A tensor without memory that says it is on device 0."""

    def get_device(self):
        return 0


@pytest.mark.parametrize("cols", [1 << 31, 1 << 32, (1 << 32) + 8])
def test_the_binding_refuses_widths_beyond_the_library(cols):
    """Cut to 32 bits, 2^32 + 8 columns would be 8."""
    x = torch.empty(1, cols, dtype=torch.bfloat16, device="meta").as_subclass(OnDevice)
    w = torch.empty(4, cols, dtype=torch.bfloat16, device="meta").as_subclass(OnDevice)
    v = torch.empty(1, device="meta").as_subclass(OnDevice)
    for call in (lambda: gn.layer_norm(x), lambda: gn.layer_norm_grad(x, x, v, v), lambda: gn.dropout(x, 0.1, 1),
                 lambda: gn.gated_ffn(x, w, w, w), lambda: gn.gated_ffn_grad(x, x, w, w, w, w, w)):
        with pytest.raises(ValueError, match="fewer than 2\\^31 columns"):
            call()
    narrow, tall = (torch.empty(*s, dtype=torch.bfloat16, device="meta").as_subclass(OnDevice) for s in ((1, 8), (cols, 8)))
    with pytest.raises(ValueError, match="fewer than 2\\^31 rows"):
        gn.gated_ffn(narrow, tall, tall, narrow)
