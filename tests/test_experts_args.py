"""Refusals of the calls of a mixture of experts: nothing is launched, so no device is needed."""
import ctypes as C
import struct

import pytest
import torch

import paper_1802_00130_b200 as gn

P = C.c_void_p(1 << 20)            # an aligned address that no refused call looks at


def refused(fn, *args):
    err = C.create_string_buffer(200)
    assert fn(*args, err, 200) == 1            # GN_EINVAL
    assert err.value
    return err.value.decode()


def router(**change):
    """gn_router as 13 words."""
    a = dict(type=1, score=0, tokens=4, experts=16, k=4, groups=4, top=2, best=2, renormalise=0, scale=1.0, logits=(1 << 20, 16), bias=0, index=1 << 20, weight=1 << 20,
             dlogits=(1 << 21, 16))
    a.update(change)
    low = lambda x: x & 0xFFFFFFFF
    words = [low(a["type"]) | a["score"] << 32, a["tokens"], low(a["experts"]) | a["k"] << 32, low(a["groups"]) | a["top"] << 32, low(a["best"]) | a["renormalise"] << 32,
             struct.unpack("q", struct.pack("d", a["scale"]))[0], *a["logits"], a["bias"], a["index"], a["weight"], *a["dlogits"]]
    return (C.c_int64 * 13)(*words)


SHARED = [(dict(type=3), "type"), (dict(type=-1), "type"), (dict(score=2), "score"), (dict(score=-1), "score"), (dict(tokens=-1), "tokens"), (dict(tokens=1 << 31), "tokens"),
          (dict(experts=0), "experts"), (dict(experts=1025), "experts"), (dict(k=0), "k must"), (dict(k=33, experts=64), "k must"), (dict(k=17), "k must"), (dict(k=-1), "k must"),
          (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(scale=1e39), "scale"), (dict(logits=(0, 16)), "logits"), (dict(logits=(1 << 20, 15)), "logits"),
          (dict(logits=(3, 16)), "logits"), (dict(index=0), "index"), (dict(index=2), "index"), (dict(weight=0), "weight"), (dict(weight=6), "weight")]


@pytest.mark.parametrize("change,word", SHARED + [
    (dict(groups=0), "groups"), (dict(groups=3), "groups"), (dict(groups=33, experts=33), "groups"), (dict(top=0), "top_groups"), (dict(top=5), "top_groups"),
    (dict(best=0), "group_best"), (dict(best=3), "group_best"), (dict(k=9), "k must"), (dict(bias=6), "bias")])
def test_route_refuses(change, word):
    assert word in refused(gn.lib().gn_route, router(**change), None)


@pytest.mark.parametrize("change,word", SHARED + [(dict(dlogits=(0, 16)), "dlogits"), (dict(dlogits=(1 << 21, 15)), "dlogits"), (dict(dlogits=(1 << 20, 16)), "place")])
def test_route_grad_refuses(change, word):
    assert word in refused(gn.lib().gn_route_grad, router(**change), None)


def test_no_arguments():
    for fn in (gn.lib().gn_route, gn.lib().gn_route_grad):
        assert "no arguments" in refused(fn, None, None)


def test_the_binding_refuses_tensors_that_are_not_on_a_device():
    x = torch.zeros(4, 8)
    for call in (lambda: gn.route(x, 2), lambda: gn.route_grad(x, x, x)):
        with pytest.raises(TypeError, match="CUDA"):
            call()


def mixture(**change):
    """gn_mixture as 39 words."""
    mats, stacks = ["x", "y", "gate", "up", "dy", "dx"], ["w_gate", "w_up", "w_down", "dw_gate", "dw_up", "dw_down"]
    a = dict(type=1, act=1, tokens=4, cols=8, inner=16, experts=3, k=2, index=1 << 20, weight=1 << 20, dweight=1 << 20)
    a.update({n: (1 << (21 + i), 16) for i, n in enumerate(mats)})
    a.update({n: (1 << (30 + i), 16, 256) for i, n in enumerate(stacks)})
    a.update(change)
    words = [a["type"] | a["act"] << 32, a["tokens"], a["cols"] | a["inner"] << 32, a["experts"] | a["k"] << 32, a["index"], a["weight"], a["dweight"]]
    words += [v for n in mats for v in a[n]] + [v for n in stacks for v in a[n]]
    return (C.c_int64 * 37)(*words)


BOTH = [(dict(type=5), "type"), (dict(act=5), "act"), (dict(tokens=-1), "tokens"), (dict(tokens=1 << 27), "tokens"), (dict(cols=0), "cols"), (dict(inner=0), "cols"),
        (dict(cols=(1 << 20) + 1), "cols"), (dict(cols=1 << 16, inner=1 << 15), "product"), (dict(experts=0), "experts"), (dict(experts=1025), "experts"), (dict(k=0), "k must"),
        (dict(k=33), "k must"), (dict(index=0), "index"), (dict(index=2), "index"), (dict(weight=0), "weight"), (dict(weight=6), "weight"), (dict(x=(0, 16)), "x:"),
        (dict(x=(1 << 20, 7)), "x:"), (dict(w_gate=(0, 8, 256)), "w_gate"), (dict(w_up=(1 << 20, 7, 256)), "w_up"), (dict(w_down=(1 << 20, 15, 256)), "w_down"),
        (dict(w_gate=(1 << 20, 8, 127)), "w_gate"), (dict(w_down=(1 << 20, 16, 127)), "w_down"), (dict(gate=(1 << 20, 15)), "gate"), (dict(up=(3, 16)), "up")]


@pytest.mark.parametrize("change,word", BOTH + [(dict(y=(0, 8)), "y:"), (dict(y=(1 << 20, 7)), "y:")])
def test_experts_refuse(change, word):
    args = mixture(**change)
    assert word in refused(gn.lib().gn_experts, args, P, 1 << 40, None)
    assert gn.lib().gn_experts_workspace(args, 0) < 0


@pytest.mark.parametrize("change,word", BOTH + [
    (dict(gate=(0, 16)), "gate"), (dict(up=(0, 16)), "up"), (dict(dy=(0, 8)), "dy"), (dict(dx=(1 << 20, 7)), "dx"), (dict(dweight=6), "dweight"),
    (dict(dw_gate=(1 << 20, 7, 256)), "dw_gate"), (dict(dw_up=(1, 16, 256)), "dw_up"), (dict(dw_down=(1 << 20, 15, 256)), "dw_down"), (dict(dw_down=(1 << 20, 16, 100)), "dw_down")])
def test_experts_grad_refuses(change, word):
    args = mixture(**change)
    assert word in refused(gn.lib().gn_experts_grad, args, P, 1 << 40, None)
    assert gn.lib().gn_experts_workspace(args, 1) < 0


@pytest.mark.parametrize("fn", ["gn_experts", "gn_experts_grad"])
@pytest.mark.parametrize("type", [0, 1, 2])
def test_experts_refuse_a_bad_workspace(fn, type):
    args = mixture(type=type)
    need = gn.lib().gn_experts_workspace(args, fn.endswith("grad"))
    assert need > 0
    for ws, n in ((None, need), (C.c_void_p((1 << 20) + 8), need), (P, need - 1)):
        assert "workspace" in refused(getattr(gn.lib(), fn), args, ws, n, None)
    assert "no arguments" in refused(getattr(gn.lib(), fn), None, P, need, None)


def test_experts_without_a_device():
    x, i, w = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(3, 16, 8)
    for call in (lambda: gn.experts(x, i, x[:, :2], w, w, w), lambda: gn.experts_grad(x, x, i, x[:, :2], x, x, w, w, w)):
        with pytest.raises(TypeError, match="CUDA"):
            call()


def layout(fn, **change):
    a = dict(type=1, experts=2, rows=20, cols=40, group=32, w=P, ld=40, stride=800, scales=P, q=P, scale=P, st=None)
    a.update(change)
    if fn == "gn_quantize4":
        del a["scales"]
    if fn == "gn_unpack4":
        a = dict(type=a["type"], experts=a["experts"], rows=a["rows"], cols=a["cols"], group=a["group"], q=a["q"], scale=a["scale"], w=a["w"], ld=a["ld"], stride=a["stride"], st=None)
    return refused(getattr(gn.lib(), fn), *a.values())


SIZES4 = [(dict(type=3), "type"), (dict(experts=0), "experts"), (dict(experts=1025), "experts"), (dict(rows=0), "rows"), (dict(cols=0), "rows"), (dict(rows=1 << 16, cols=1 << 15), "rows"),
          (dict(cols=(1 << 20) + 1), "rows"), (dict(group=16), "group"), (dict(group=256), "group")]


@pytest.mark.parametrize("fn", ["gn_pack4", "gn_quantize4", "gn_unpack4"])
@pytest.mark.parametrize("change,word", SIZES4 + [(dict(w=None), "weights"), (dict(ld=39), "weights"), (dict(stride=799), "weights"), (dict(q=None), "packed"), (dict(scale=C.c_void_p(8)), "packed")])
def test_layouts_refuse(fn, change, word):
    assert word in layout(fn, **change)


def test_layouts_refuse_misaligned_elements():
    assert "scales" in layout("gn_pack4", scales=C.c_void_p(3)) and "scales" in layout("gn_pack4", scales=None)
    assert "weights" in layout("gn_quantize4", w=C.c_void_p(3)) and "weights" in layout("gn_unpack4", w=C.c_void_p(3))
    lib = gn.lib()
    assert lib.gn_weight4_bytes(0, 16, 16) < 0 and lib.gn_weight4_scales(1, 16, 16, 48) < 0 and lib.gn_weight4_bytes(1, 1 << 20, 1 << 11) < 0
    assert lib.gn_weight4_bytes(2, 17, 129) == 2 * 2 * 2 * 1024 and lib.gn_weight4_scales(2, 17, 129, 32) == 2 * 2 * 2 * 64


@pytest.mark.parametrize("change,word", [c for c in SIZES4 if "experts" not in c[0]] + [
    (dict(tokens=-1), "tokens"), (dict(tokens=1 << 20), "tokens"), (dict(x=None), "x:"), (dict(ldx=39), "x:"), (dict(q=C.c_void_p(8)), "packed"), (dict(y=None), "y:"), (dict(ldy=19), "y:"),
    (dict(type=0, ws=None), "workspace"), (dict(type=0, ws=C.c_void_p(8)), "workspace"), (dict(type=0, n=719), "workspace")])
def test_matvec4_refuses(change, word):
    a = dict(type=1, tokens=3, rows=20, cols=40, group=32, x=P, ldx=40, q=P, scale=P, y=P, ldy=20, ws=P, n=1 << 30, st=None)
    a.update(change)
    assert word in refused(gn.lib().gn_matvec4, *a.values())


def ffn4(**change):
    """gn_ffn4 as 17 words."""
    a = dict(type=1, act=1, tokens=4, cols=8, inner=16, experts=3, k=2, group=32, index=1 << 20, weight=1 << 20, x=(1 << 21, 8), y=(1 << 22, 8))
    a.update({n: 1 << 23 for n in ("q_gate", "s_gate", "q_up", "s_up", "q_down", "s_down")})
    a.update(change)
    words = [a["type"] | a["act"] << 32, a["tokens"], a["cols"] | a["inner"] << 32, a["experts"] | a["k"] << 32, a["group"], a["index"], a["weight"], *a["x"], *a["y"]]
    return (C.c_int64 * 17)(*words, *(a[n] for n in ("q_gate", "s_gate", "q_up", "s_up", "q_down", "s_down")))


@pytest.mark.parametrize("change,word", [
    (dict(type=4), "type"), (dict(act=7), "act"), (dict(tokens=-1), "tokens"), (dict(tokens=1 << 19), "tokens"), (dict(cols=0), "rows"), (dict(inner=0), "rows"), (dict(experts=0), "experts"),
    (dict(k=0), "k must"), (dict(k=33), "k must"), (dict(group=1), "group"), (dict(index=0), "index"), (dict(index=0, experts=1), "index"), (dict(index=2), "index"), (dict(weight=0), "weight"),
    (dict(x=(0, 8)), "x:"), (dict(x=(1 << 21, 7)), "x:"), (dict(y=(0, 8)), "y:"), (dict(y=(1 << 21, 7)), "y:"), (dict(q_gate=0), "packed"), (dict(s_up=8), "packed"), (dict(q_down=4), "packed")])
def test_gated_ffn4_refuses(change, word):
    args = ffn4(**change)
    assert word in refused(gn.lib().gn_gated_ffn4, args, P, 1 << 40, None)
    assert gn.lib().gn_gated_ffn4_workspace(args) < 0


def test_gated_ffn4_refuses_a_bad_workspace():
    args = ffn4()
    need = gn.lib().gn_gated_ffn4_workspace(args)
    assert need > 0
    for ws, n in ((None, need), (C.c_void_p((1 << 20) + 8), need), (P, need - 1)):
        assert "workspace" in refused(gn.lib().gn_gated_ffn4, args, ws, n, None)
    assert "no arguments" in refused(gn.lib().gn_gated_ffn4, None, P, need, None)


def test_4_bit_weights_without_a_device():
    q = torch.zeros(4, 8, dtype=torch.uint8)
    for call in (lambda: gn.pack4(q, q.float()), lambda: gn.quantize4(q.float())):
        with pytest.raises(TypeError, match="CUDA"):
            call()


def test_4_bit_calls_take_fewer_than_2_to_the_19_tokens():
    """Their tiles are the second dimension of a grid: what is taken fits, whatever the type."""
    lib, most = gn.lib(), 1 << 19
    for type in (0, 1, 2):
        assert lib.gn_matvec4_workspace(type, most - 1, 40, P, 40) >= 0 and lib.gn_matvec4_workspace(type, most, 40, P, 40) < 0
        assert "tokens" in refused(lib.gn_matvec4, type, most, 20, 40, 32, P, 40, P, P, P, 20, P, 1 << 40, None)
        for k in (1, 2):
            assert lib.gn_gated_ffn4_workspace(ffn4(type=type, k=k, tokens=most // k - 1)) > 0 and lib.gn_gated_ffn4_workspace(ffn4(type=type, k=k, tokens=most // k)) < 0


def test_4_bit_weights_have_the_bytes_of_their_sizes():
    q, scale = torch.zeros(2 * 2 * 1024, dtype=torch.uint8), torch.zeros(2 * 2 * 64)
    w = gn.Weight4(q, scale, None, 17, 129, 32)
    assert w.shape == (17, 129) and gn.Weight4(q, scale, 2, 16, 129, 32).shape == (2, 16, 129)
    for bad in ((q[1:], scale, None, 17, 129, 32), (q, scale[1:], None, 17, 129, 32), (q, scale, None, 33, 129, 32), (q, scale, None, 17, 257, 32), (q, scale, 2, 17, 129, 32), (q, scale, None, 17, 129, 64),
                (q, scale, None, 17, 129, 48), (q, scale, None, 0, 129, 32), (q, scale, 0, 17, 129, 32), (q, scale, None, 1 << 40, 129, 32), (torch.zeros(4096, 2, dtype=torch.uint8)[:, 0], scale, None, 17, 129, 32)):
        with pytest.raises(ValueError):
            gn.Weight4(*bad)
    for bad in ((q.int(), scale, None, 17, 129, 32), (q, scale.double(), None, 17, 129, 32), (q, None, None, 17, 129, 32), (q, scale, None, 17.0, 129, 32), (q, scale, 1.0, 17, 129, 32)):
        with pytest.raises(TypeError):
            gn.Weight4(*bad)
    with pytest.raises(TypeError, match="CUDA"):
        gn.unpack4(w)
