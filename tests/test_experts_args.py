"""Refusals of the calls of a mixture of experts: nothing is launched, so no device is needed."""
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


def route(**change):
    a = dict(type=1, score=0, tokens=4, experts=16, k=4, logits=P, ld=16, bias=None, groups=4, top=2, best=2, renormalise=0, scale=1.0, index=P, weight=P, st=None)
    a.update(change)
    return refused(gn.lib().gn_route, *a.values())


SHARED = [(dict(type=3), "type"), (dict(score=2), "score"), (dict(score=-1), "score"), (dict(tokens=-1), "tokens"), (dict(tokens=1 << 31), "tokens"), (dict(experts=0), "experts"),
          (dict(experts=1025), "experts"), (dict(k=0), "k must"), (dict(k=33, experts=64), "k must"), (dict(k=17), "k must"), (dict(scale=float("nan")), "scale"),
          (dict(scale=float("inf")), "scale"), (dict(scale=1e39), "scale"), (dict(logits=None), "logits"), (dict(ld=15), "logits"), (dict(logits=C.c_void_p(3)), "logits"),
          (dict(index=None), "index"), (dict(index=C.c_void_p(2)), "index")]


@pytest.mark.parametrize("change,word", SHARED + [
    (dict(groups=0), "groups"), (dict(groups=3), "groups"), (dict(groups=33, experts=33), "groups"), (dict(top=0), "top_groups"), (dict(top=5), "top_groups"),
    (dict(best=0), "group_best"), (dict(best=3), "group_best"), (dict(k=9), "k must"), (dict(bias=C.c_void_p(6)), "bias"), (dict(weight=None), "weight"),
    (dict(weight=C.c_void_p(6)), "weight")])
def test_route_refuses(change, word):
    assert word in route(**change)


def route_grad(**change):
    a = dict(type=1, score=0, tokens=4, experts=16, k=4, dweight=P, logits=P, ld=16, index=P, renormalise=0, scale=1.0, dlogits=C.c_void_p(1 << 21), ld_d=16, st=None)
    a.update(change)
    return refused(gn.lib().gn_route_grad, *a.values())


@pytest.mark.parametrize("change,word", SHARED + [(dict(dweight=None), "dweight"), (dict(dlogits=None), "dlogits"), (dict(ld_d=15), "dlogits"), (dict(dlogits=P), "place")])
def test_route_grad_refuses(change, word):
    assert word in route_grad(**change)


def test_the_binding_refuses_tensors_that_are_not_on_a_device():
    x = torch.zeros(4, 8)
    for call in (lambda: gn.route(x, 2), lambda: gn.route_grad(x, x, x)):
        with pytest.raises(TypeError, match="CUDA"):
            call()
