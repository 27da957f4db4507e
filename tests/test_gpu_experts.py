"""A mixture's experts and their backward pass against a plain form in 64 bits."""
import math

import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import TYPES, act64, rand, u, within
from mixture_common import check_experts, check_experts_grad, choices, used, weights_of

pytestmark = pytest.mark.gpu

ACTS = ["sigmoid", "silu", "gelu", "gelu_tanh", "relu"]
# tokens, cols, inner, experts, k: single tokens, odd sizes, tile edges, experts without tokens, one expert, several tiles of an expert
SHAPES = [(1, 1, 1, 1, 1), (1, 64, 128, 4, 2), (2, 8, 16, 2, 2), (3, 7, 5, 3, 3), (1, 1000, 333, 9, 8), (16, 256, 512, 8, 4), (40, 136, 72, 64, 8), (5, 64, 64, 300, 4),
          (63, 72, 65, 1, 1), (64, 64, 256, 1, 1), (65, 264, 129, 1, 1), (129, 617, 301, 3, 2), (300, 264, 520, 5, 2), (1003, 200, 333, 7, 3), (700, 128, 256, 2, 1), (2000, 96, 40, 33, 6),
          (513, 33, 130, 1024, 2), (150, 520, 24, 6, 6), (4000, 40, 72, 4, 2)]


def inputs(tokens, cols, inner, experts, k, t, pad=0, seed=0):
    x = rand((tokens, cols), t, seed + 1, pad=pad)
    return (x, *choices(tokens, experts, k, seed), weights_of(experts, cols, inner, t, seed, pad))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(t, shape):
    x, index, weight, w = inputs(*shape, TYPES[t])
    for i, save in enumerate((False, True)):
        act = ACTS[(sum(shape) + i) % 5]
        check_experts(gn.experts(x, index, weight, *w, act, save=save), x, index, weight, w, act, TYPES[t])
    gn.gated_ffn_status()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(t, shape):
    x, index, weight, w = inputs(*shape, TYPES[t])
    act = ACTS[sum(shape) % 5]
    _, gate, up = gn.experts(x, index, weight, *w, act, save=True)
    dy = rand(x.shape, TYPES[t], 9, 0.3)
    check_experts_grad(gn.experts_grad(dy, x, index, weight, gate, up, *w, act), dy, x, index, weight, gate, up, w, act, TYPES[t])
    gn.gated_ffn_status()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_strides(t, pad):
    x, index, weight, w = inputs(90, 72, 40, 5, 2, TYPES[t], pad)
    got = gn.experts(x, index, weight, *w, "silu", save=True)
    check_experts(got, x, index, weight, w, "silu", TYPES[t])
    dy, gate, up = (rand(s, TYPES[t], 9, 0.3, pad=pad) for s in ((90, 72), (180, 40), (180, 40)))
    check_experts_grad(gn.experts_grad(dy, x, index, weight, gate, up, *w, "silu"), dy, x, index, weight, gate, up, w, "silu", TYPES[t])


@pytest.mark.parametrize("t", TYPES)
def test_choices_of_all_kinds(t):
    """All tokens with one expert, the same expert twice, no expert at all, indices far out."""
    x, index, weight, w = inputs(130, 64, 48, 6, 3, TYPES[t])
    dy = rand(x.shape, TYPES[t], 9, 0.3)
    doubtful = index.clone()
    doubtful[::3] = -1
    doubtful[1::5, 1] = 6
    doubtful[2::7, 2] = 2 ** 31 - 1
    doubtful[5] = -2 ** 31
    for table in (torch.full_like(index, 4), torch.zeros_like(index), index[:, :1].expand(-1, 3).contiguous(), doubtful, torch.full_like(index, -1)):
        got = gn.experts(x, table, weight, *w, "gelu", save=True)
        check_experts(got, x, table, weight, w, "gelu", TYPES[t])
        grads = gn.experts_grad(dy, x, table, weight, *got[1:], *w, "gelu")
        check_experts_grad(grads, dy, x, table, weight, *got[1:], w, "gelu", TYPES[t])
        none = (table < 0) | (table >= 6)
        assert bool((grads[1][none] == 0).all()) and bool((got[0][none.all(1)] == 0).all()) and bool((grads[0][none.all(1)] == 0).all())


@pytest.mark.parametrize("t", TYPES)
def test_an_expert_is_untouched_by_another_ones_nan(t):
    x, index, weight, w = inputs(70, 72, 40, 4, 1, TYPES[t])
    dy = rand(x.shape, TYPES[t], 9, 0.3)
    y, gate, up = gn.experts(x, index, weight, *w, save=True)
    grads = gn.experts_grad(dy, x, index, weight, gate, up, *w)
    w = [m.clone() for m in w]
    for m in w:
        m[2] = math.nan
    index = index.clone()
    x, dy = x.clone(), dy.clone()
    x[index[:, 0] == 3] = math.inf
    dy[index[:, 0] == 3] = math.nan
    keep = ((index != 2) & (index != 3))[:, 0]
    y2, gate2, up2 = gn.experts(x, index, weight, *w, save=True)
    grads2 = gn.experts_grad(dy, x, index, weight, gate2, up2, *w)
    assert torch.equal(y[keep], y2[keep]) and torch.equal(grads[0][keep], grads2[0][keep]) and torch.equal(grads[1][keep], grads2[1][keep])
    for a, b in zip(grads[2:], grads2[2:]):
        assert torch.equal(a[:2], b[:2])


def test_gradient_is_that_of_differences():
    """Central differences of the 64-bit form at step h, in FP32: products off by 1e-5 of what they add up, differences by h^2."""
    x, index, weight, w = inputs(5, 6, 4, 3, 2, torch.float32)
    dy = rand((5, 6), torch.float32, 9)
    _, gate, up = gn.experts(x, index, weight, *w, "gelu", save=True)
    got = gn.experts_grad(dy, x, index, weight, gate, up, *w, "gelu")

    def f(x, s, wg, wu, wd):
        y = torch.zeros_like(x)
        for e, t, j in used(index, 3):
            y.index_put_((t,), s[t, j][:, None] * ((act64("gelu", x[t] @ wg[e].T)[0] * (x[t] @ wu[e].T)) @ wd[e].T), accumulate=True)
        return (y * dy.double()).sum()

    args = [x.double(), weight.double(), *(m.double() for m in w)]
    h = 1e-5
    for n, g in enumerate(got):
        flat, want = args[n].view(-1), torch.empty(args[n].numel(), dtype=torch.float64, device="cuda")
        for i in range(flat.numel()):
            keep = flat[i].clone()
            flat[i] = keep + h
            hi = f(*args)
            flat[i] = keep - h
            want[i] = (hi - f(*args)) / (2 * h)
            flat[i] = keep
        within(g.reshape(-1), want, torch.full_like(want, 1e-4), f"output {n}")


@pytest.mark.parametrize("t", TYPES)
def test_same_bits_again_on_another_stream_and_captured(t):
    x, index, weight, w = inputs(300, 264, 136, 6, 2, TYPES[t])
    dy = rand(x.shape, TYPES[t], 9, 0.3)

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
    new_index, new_weight = choices(300, 6, 2, 5)
    index.copy_(new_index)
    weight.copy_(new_weight)
    x.copy_(rand(x.shape, TYPES[t], 77))
    for g in graphs:
        g.replay()
    plain = both()
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(out, plain))


@pytest.mark.parametrize("t", TYPES)
def test_no_tokens(t):
    x, index, weight, w = inputs(4, 16, 24, 3, 2, TYPES[t])
    y, gate, up = gn.experts(x[:0], index[:0], weight[:0], *w, save=True)
    assert y.shape == (0, 16) and gate.shape == (0, 24)
    grads = gn.experts_grad(x[:0], x[:0], index[:0], weight[:0], gate, up, *w)
    assert grads[0].shape == (0, 16) and grads[1].shape == (0, 2) and all(bool((g == 0).all()) for g in grads[2:])


def test_refusals():
    x, index, weight, w = inputs(8, 16, 24, 3, 2, torch.bfloat16)
    for call in (lambda: gn.experts(x, index[:7], weight, *w), lambda: gn.experts(x, index, weight[:, :1], *w), lambda: gn.experts(x, index, weight, w[0][:2], w[1], w[2]),
                 lambda: gn.experts(x, index, weight, w[0], w[1], w[2].transpose(1, 2)), lambda: gn.experts(x, index, weight, *w, "tanh"),
                 lambda: gn.experts(x, index, weight, w[0][0], w[1], w[2]), lambda: gn.experts(x, index, weight, w[0][:1].expand(3, -1, -1), w[1], w[2]),
                 lambda: gn.experts(x, index.t().contiguous().t(), weight, *w)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gn.experts(x, index.long(), weight, *w), lambda: gn.experts(x, index, weight.to(torch.bfloat16), *w), lambda: gn.experts(x, index, weight, w[0].float(), w[1], w[2]),
                 lambda: gn.experts(x.double(), index, weight, *w), lambda: gn.experts(x, index, weight, w[0].cpu(), w[1], w[2])):
        with pytest.raises(TypeError):
            call()
    many = torch.zeros(8, 33, device="cuda", dtype=torch.int32)
    with pytest.raises(gn.GnError):
        gn.experts(x, many, many.float(), *w)
