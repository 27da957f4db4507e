"""A mixture's experts in FP32 in each of their three forms, which sizes choose: small and large tiles on FMAs, and the tensor cores on operands in three parts."""
import math

import pytest
import torch

import paper_1802_00130_b200 as gn
from expert_paths import BACKWARD, FORWARD, path
from feedforward_common import rand
from mixture_common import check_experts, check_experts_grad, choices, weights_of

pytestmark = pytest.mark.gpu
F32 = torch.float32
ACTS = ["sigmoid", "silu", "gelu", "gelu_tanh", "relu"]
# for each form a size that takes it forward and backward
BOTH = [("small", (300, 264, 136, 6, 2)), ("large", (700, 265, 129, 300, 1)), ("large", (4000, 120, 30, 512, 4)), ("tensor", (700, 200, 333, 6, 3)), ("tensor", (400, 264, 520, 3, 2))]


def inputs(tokens, cols, inner, experts, k, pad=0, seed=0):
    x = rand((tokens, cols), F32, seed + 1, pad=pad)
    return (x, *choices(tokens, experts, k, seed), weights_of(experts, cols, inner, F32, seed, pad))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("name,shape", [(n, s) for n in FORWARD for s in FORWARD[n]])
def test_forward(name, shape, act):
    assert path(*shape, False) == name
    x, index, weight, w = inputs(*shape)
    check_experts(gn.experts(x, index, weight, *w, act, save=True), x, index, weight, w, act, F32)
    gn.gated_ffn_status()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("name,shape", [(n, s) for n in BACKWARD for s in BACKWARD[n]])
def test_backward(name, shape, act):
    assert path(*shape, True) == name
    x, index, weight, w = inputs(*shape)
    _, gate, up = gn.experts(x, index, weight, *w, act, save=True)
    dy = rand(x.shape, F32, 9, 0.3)
    check_experts_grad(gn.experts_grad(dy, x, index, weight, gate, up, *w, act), dy, x, index, weight, gate, up, w, act, F32)
    gn.gated_ffn_status()


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("name,shape", BOTH)
def test_strides(name, shape, pad):
    assert path(*shape, False) == path(*shape, True) == name
    x, index, weight, w = inputs(*shape, pad=pad)
    check_experts(gn.experts(x, index, weight, *w, "silu", save=True), x, index, weight, w, "silu", F32)
    pairs, inner = shape[0] * shape[4], shape[2]
    dy, gate, up = (rand(s, F32, 9, 0.3, pad=pad) for s in (x.shape, (pairs, inner), (pairs, inner)))
    check_experts_grad(gn.experts_grad(dy, x, index, weight, gate, up, *w, "silu"), dy, x, index, weight, gate, up, w, "silu", F32)


@pytest.mark.parametrize("name,shape", BOTH)
def test_choices_of_all_kinds(name, shape):
    """All tokens with one expert, the same expert twice, no expert at all, indices far out, most experts without a token."""
    x, index, weight, w = inputs(*shape)
    n, k = shape[3], shape[4]
    dy = rand(x.shape, F32, 9, 0.3)
    doubtful = index.clone()
    doubtful[::3] = -1
    doubtful[1::5, k - 1] = n
    doubtful[2::7, 0] = 2 ** 31 - 1
    doubtful[5] = -2 ** 31
    few = index % 2
    for table in (torch.full_like(index, n - 1), torch.zeros_like(index), index[:, :1].expand(-1, k).contiguous(), doubtful, few, torch.full_like(index, -1)):
        got = gn.experts(x, table, weight, *w, "gelu", save=True)
        check_experts(got, x, table, weight, w, "gelu", F32)
        grads = gn.experts_grad(dy, x, table, weight, *got[1:], *w, "gelu")
        check_experts_grad(grads, dy, x, table, weight, *got[1:], w, "gelu", F32)
        none = (table < 0) | (table >= n)
        assert bool((grads[1][none] == 0).all()) and bool((got[0][none.all(1)] == 0).all()) and bool((grads[0][none.all(1)] == 0).all())
        empty = torch.ones(n, dtype=torch.bool, device="cuda")
        empty[table[~none].long().unique()] = False
        assert all(bool((g[empty] == 0).all()) for g in grads[2:])


@pytest.mark.parametrize("name,shape", BOTH)
def test_an_expert_is_untouched_by_another_ones_nan(name, shape):
    x, index, weight, w = inputs(*shape)
    index = index.clone()
    index[:] = index[:, :1]                                  # (a token is one expert's, so that what is to be left alone is whole tokens)
    bad_w, bad_x = 1, 2
    if shape[3] > 100:                                       # (an even share for few experts: several rows each)
        index %= 20
    dy = rand(x.shape, F32, 9, 0.3)
    y, gate, up = gn.experts(x, index, weight, *w, save=True)
    grads = gn.experts_grad(dy, x, index, weight, gate, up, *w)
    w = [m.clone() for m in w]
    for m in w:
        m[bad_w] = math.nan
    x, dy = x.clone(), dy.clone()
    x[index[:, 0] == bad_x] = math.inf
    dy[index[:, 0] == bad_x] = math.nan
    keep = (index[:, 0] != bad_w) & (index[:, 0] != bad_x)
    assert 10 < int(keep.sum()) < shape[0] - 10
    y2, gate2, up2 = gn.experts(x, index, weight, *w, save=True)
    grads2 = gn.experts_grad(dy, x, index, weight, gate2, up2, *w)
    assert torch.equal(y[keep], y2[keep]) and torch.equal(grads[0][keep], grads2[0][keep]) and torch.equal(grads[1][keep], grads2[1][keep])
    assert not bool(y2[~keep].isfinite().all(1).any())
    others = [e for e in range(shape[3]) if e not in (bad_w, bad_x)]
    for a, b in zip(grads[2:], grads2[2:]):
        assert torch.equal(a[others], b[others])


@pytest.mark.parametrize("name,shape", BOTH)
def test_same_bits_again_on_another_stream_and_captured(name, shape):
    x, index, weight, w = inputs(*shape)
    dy = rand(x.shape, F32, 9, 0.3)

    def both(stream=None):
        y, gate, up = gn.experts(x, index, weight, *w, save=True, stream=stream)
        return [y, *gn.experts_grad(dy, x, index, weight, gate, up, *w, stream=stream)]

    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other, again = both(side), both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(first, other, again))
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(both())
    new_index, new_weight = choices(shape[0], shape[3], shape[4], 5)
    index.copy_(new_index)
    weight.copy_(new_weight)
    x.copy_(rand(x.shape, F32, 77))
    for g in graphs:
        g.replay()
    plain = both()
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(out, plain))
