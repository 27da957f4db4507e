"""Routing to experts against the definition in 64 bits: orders have to be equal, weights and gradients are within FP32's roundings."""
import math

import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import E, TYPES, rand, tiny, u, within

pytestmark = pytest.mark.gpu
INF = math.inf


def scores64(logits, score):
    z = logits.double()
    if score == "sigmoid":
        return torch.special.expit(z)
    return torch.where((z == -INF).all(1, keepdim=True), 0.0, torch.softmax(z, 1))


def largest(v, k):
    """The k largest of a row, ties by number, NaN behind everything."""
    v = torch.where(v.isnan(), -1e306, torch.where(v == -INF, -1e305, v))
    return v.sort(dim=1, descending=True, stable=True).indices[:, :k]


def route64(logits, k, score, bias, groups, top, best, renormalise, scale, even=False):
    s, z = scores64(logits, score), logits.double()
    value = s if bias is None else s + bias.double()
    order = z if bias is None else value
    T, n = z.shape
    clear = torch.ones(T, dtype=torch.bool, device="cuda")
    if groups > 1:
        each = n // groups
        g = order.view(T, groups, each).amax(2)
        if best == 2:                # (scores and biases each by themselves: the same ones in other pairs are the same sum, without a rounding that might differ)
            two = value.view(T, groups, each).sort(dim=2, descending=True).indices[:, :, :2]
            g = s.view(T, groups, each).gather(2, two).sum(2)
            if bias is not None:
                g = g + bias.double().view(1, groups, each).expand(T, groups, each).gather(2, two).sum(2)
        # Sums of scores that lie nearer than 64 bits tell apart: exp(x + 2d) + exp(x) is larger than 2 exp(x + d) by exp(x) d^2, at d = 2e-8 4e-16 of it, and
        # each of the four exponentials, their division by the sum and the addition are off by up to 2^-53 = 1.1e-16 of them and more, here as there.
        if top < groups:
            v = g.sort(dim=1, descending=True).values
            clear = ~((v[:, top - 1] - v[:, top]).abs() <= 16 * 2.0 ** -53 * v[:, top].abs())
            if even or best == 1:    # (equal because they are the same numbers)
                clear |= v[:, top - 1] == v[:, top]
        kept = torch.zeros(T, groups, dtype=torch.bool, device="cuda").scatter_(1, largest(g, top), True).repeat_interleave(each, 1)
        order = torch.where(kept, torch.where(order == -INF, -1e305, order), -1e307)
    index = largest(order, k)
    w = s.gather(1, index)
    if renormalise:
        total = w.sum(1, keepdim=True)
        w = w / total.masked_fill(total == 0, 1)
    return index, w * scale, clear


# A score: see the bound in the kernel (150 steps of 2^-24); a sum of k of them and the division: 40 more; the scale's product 1.
W = 200 * E


def check(logits, k, score="softmax", bias=None, groups=1, top=1, best=1, renormalise=False, scale=1.0, even=False):
    index, weight = gn.route(logits, k, score, bias, groups, top, best, renormalise, scale)
    ref, w, clear = route64(logits, k, score, bias, groups, top, best, renormalise, scale, even)
    assert torch.equal(index[clear].long(), ref[clear])
    within(weight[clear], w[clear], w[clear].abs() * 2 * W + 1e-37, "weight")
    assert bool((index >= 0).all()) and bool((index < logits.shape[1]).all())
    return index, weight


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,experts,k", [(1, 1, 1), (1, 2, 2), (3, 7, 7), (17, 31, 4), (5, 32, 32), (4, 33, 1), (301, 60, 4), (1000, 64, 6), (77, 128, 8), (2049, 256, 8),
                                              (63, 257, 5), (9, 512, 16), (9, 1000, 32), (5, 1024, 3)])
def test_choice_and_weights(t, tokens, experts, k):
    logits = rand((tokens, experts), TYPES[t], tokens + experts, 1.5)
    bias = rand((1, experts), torch.float32, 5, 0.1)[0].contiguous()
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            check(logits, k, score, None, renormalise=renormalise)
            check(logits, k, score, bias, renormalise=renormalise, scale=2.5)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("experts,groups,top,k", [(8, 4, 2, 3), (64, 8, 3, 6), (256, 8, 4, 8), (60, 4, 1, 15), (96, 32, 5, 7), (32, 32, 4, 4), (512, 2, 1, 9), (1024, 32, 31, 8)])
def test_groups(t, experts, groups, top, k):
    logits = rand((513, experts), TYPES[t], experts, 1.5)
    bias = rand((1, experts), torch.float32, 5, 0.1)[0].contiguous()
    for score in ("softmax", "sigmoid"):
        for best in (1, 2):
            check(logits, k, score, None, groups, top, best, True)
            check(logits, k, score, bias, groups, top, best, False, 1.5)


@pytest.mark.parametrize("experts,groups", [(16, 1), (256, 1), (256, 8), (1024, 8)])
def test_values_that_fp32_cannot_tell_apart(experts, groups):
    """Scores and biases whose sums differ by less than FP32's steps: the order is that of 64 bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    logits = torch.randint(-2, 3, (400, experts), generator=g, device="cuda").float() * 1e-3 + torch.randint(0, 3, (400, experts), generator=g, device="cuda") * 2e-8
    bias = torch.randint(0, 4, (experts,), generator=g, device="cuda").float() * 6e-8
    for score in ("softmax", "sigmoid"):
        for best in (1, 2):
            check(logits, 8, score, bias, groups, max(1, groups // 2), best)
            check(logits, 8, score, None, groups, max(1, groups // 2), best)


@pytest.mark.parametrize("bias", [None, 0.0, 0.25])
@pytest.mark.parametrize("groups", [1, 4])
def test_equal_values_go_by_number(bias, groups):
    logits = torch.zeros(5, 64, device="cuda", dtype=torch.bfloat16)
    logits[1] = 3.0
    logits[2, 40:] = 1.0
    logits[3, ::2] = -0.0
    logits[4] = rand((1, 64), torch.float32, 1).sign()[0].to(torch.bfloat16)
    b = None if bias is None else torch.full((64,), bias, device="cuda")
    for k in (1, 8, 16):
        for score in ("softmax", "sigmoid"):
            for best in (1, 2):
                check(logits, k, score, b, groups, 1, best, even=True)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("groups", [1, 4])
def test_masked_experts(t, with_bias, groups):
    logits = rand((200, 64), TYPES[t], 7, 1.5)
    logits[torch.rand(200, 64, device="cuda") < 0.9] = -INF
    logits[3] = -INF
    logits[4] = -INF
    logits[4, 50] = 1.0
    logits[5] = torch.finfo(TYPES[t]).min                     # a mask by the lowest value: an even row
    bias = rand((1, 64), torch.float32, 5, 0.1)[0].contiguous() if with_bias else None
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            index, weight = check(logits, 16, score, bias, groups, max(1, groups // 2), 2, renormalise)
            assert bool((weight[3] == 0).all())
            assert bool((index.sort(1).values.diff(dim=1) > 0).all())


def test_experts_kept_out_by_the_bias():
    logits = rand((50, 32), torch.float32, 1)
    bias = torch.zeros(32, device="cuda")
    bias[::2] = -INF
    index, _ = check(logits, 16, "sigmoid", bias)
    assert bool((index % 2 == 1).all())


def test_nan_and_infinity():
    logits = rand((6, 40), torch.float32, 1)
    logits[0, 5] = math.nan
    logits[1] = math.nan
    logits[2, 7] = INF
    logits[3, 38:] = math.nan
    bias = torch.zeros(40, device="cuda")
    bias[3] = math.nan
    for b in (None, bias):
        for groups in (1, 8):
            for k in (4, 32 // groups):
                index, weight = gn.route(logits, k, "sigmoid", b, groups, 1)
                assert bool((index >= 0).all()) and bool((index < 40).all())
                assert bool((index.sort(1).values.diff(dim=1) > 0).all())
                index, weight = gn.route(logits, k, "softmax", b, groups, 1)
                assert bool(weight[:4].isnan().all()) and bool(weight[4:].isfinite().all())
                assert bool((index >= 0).all()) and bool((index < 40).all())
    index, _ = gn.route(logits, 32, "sigmoid")
    assert 5 not in index[0].tolist() and index[1].tolist() == list(range(32)) and index[2, 0] == 7


def grad64(dweight, logits, index, score, renormalise, scale):
    z = logits.double().requires_grad_()
    s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, 1)
    w = s.gather(1, index.long())
    if renormalise:
        w = w / w.sum(1, keepdim=True)
    (w * scale).backward(dweight.double())
    return z.grad


def grad_bound(dweight, logits, index, score, scale):
    """The terms of the sums, each off by the score's 200 steps twice and by k + 8 roundings, as a sum of magnitudes."""
    s = scores64(logits, score)
    k = index.shape[1]
    mine = s.gather(1, index.long())
    a = dweight.double().abs() * abs(scale)
    per = a.amax(1, keepdim=True) * k
    out = s * per                                           # (shares and scores are no larger than s over their sum)
    total = mine.sum(1, keepdim=True).clamp(min=1e-300)
    return torch.maximum(out, out / total) * (2 * W + (k + 8) * E)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,experts,k", [(1, 1, 1), (3, 7, 7), (17, 31, 4), (5, 32, 32), (301, 60, 4), (1000, 64, 6), (2049, 256, 8), (63, 257, 5), (9, 1000, 32)])
def test_gradient(t, tokens, experts, k):
    logits = rand((tokens, experts), TYPES[t], tokens + experts, 1.5)
    dweight = rand((tokens, k), torch.float32, 2)
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            index, _ = gn.route(logits, k, score, renormalise=renormalise, scale=1.5)
            got = gn.route_grad(dweight, logits, index, score, renormalise, 1.5)
            ref = grad64(dweight, logits, index, score, renormalise, 1.5)
            assert got.dtype == TYPES[t] and got.shape == logits.shape
            within(got, ref, grad_bound(dweight, logits, index, score, 1.5) + ref.abs() * u(TYPES[t]) + tiny(TYPES[t]) + 1e-37, f"dlogits {score} {renormalise}")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_gradient_is_that_of_differences(score, renormalise):
    """Central differences of 64-bit weights at step h: an error of h^2 and of 2^-52 / h."""
    logits, dweight = rand((4, 20), torch.float32, 3), rand((4, 5), torch.float32, 4)
    index, _ = gn.route(logits, 5, score, renormalise=renormalise)
    got = gn.route_grad(dweight, logits, index, score, renormalise)

    def f(z):
        s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, 1)
        w = s.gather(1, index.long())
        return ((w / w.sum(1, keepdim=True) if renormalise else w) * dweight.double()).sum(1)

    h = 1e-5
    for e in range(20):
        d = torch.zeros(4, 20, device="cuda", dtype=torch.float64)
        d[:, e] = h
        within(got[:, e], (f(logits.double() + d) - f(logits.double() - d)) / (2 * h), torch.full((4,), 1e-5, device="cuda", dtype=torch.float64), "difference")


def test_gradient_of_masked_rows_and_of_doubtful_indices():
    logits = rand((6, 48), torch.bfloat16, 1)
    logits[0] = -INF
    logits[1, 10:] = -INF
    index = torch.arange(4, device="cuda", dtype=torch.int32).repeat(6, 1)
    index[2] = torch.tensor([5, 5, 7, 5])
    index[3] = torch.tensor([-1, 48, 2, 2 ** 31 - 1])
    index[4] = -2 ** 31
    dweight = rand((6, 4), torch.float32, 2)
    for score in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            got = gn.route_grad(dweight, logits, index, score, renormalise).double()
            assert bool((got[0] == 0).all()) and bool((got[1, 10:] == 0).all()) and bool((got[4] == 0).all()) and bool(got.isfinite().all())
    got = gn.route_grad(dweight, logits, index, "sigmoid")
    s = torch.sigmoid(logits.double())
    want = s[2, 5] * (1 - s[2, 5]) * dweight[2, [0, 1, 3]].double().sum()
    within(got[2, 5:6], want[None], want.abs()[None] * (u(torch.bfloat16) + 2 * W + 12 * E) + dweight[2].abs().sum() * 4 * E, "twice the same")


def test_strides_streams_and_graphs():
    wide = rand((33, 80), torch.float16, 1, 1.5)
    for view in (wide[:, :64], wide[:, 3:63], wide[::2, 1:61]):
        index, weight = check(view, 6)
        dweight = rand((view.shape[0], 6), torch.float32, 2)
        assert torch.equal(gn.route_grad(dweight, view, index), gn.route_grad(dweight, view.contiguous(), index))
    none, _ = gn.route(wide[:0], 4)
    assert none.shape == (0, 4) and gn.route_grad(torch.empty(0, 4, device="cuda"), wide[:0], none).shape == (0, 80)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = gn.route(wide, 4, stream=side), gn.route(wide, 4)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    logits, graph = wide.clone(), torch.cuda.CUDAGraph()
    bias = rand((1, 80), torch.float32, 5, 0.1)[0].contiguous()
    with torch.cuda.graph(graph):
        index, weight = gn.route(logits, 4, "sigmoid", bias, 8, 2, 2, True)
    for seed in (7, 8):
        logits.copy_(rand((33, 80), torch.float16, seed))
        graph.replay()
        again = gn.route(logits, 4, "sigmoid", bias, 8, 2, 2, True)
        assert torch.equal(index, again[0]) and torch.equal(weight, again[1])


def test_refusals():
    logits = rand((8, 16), torch.float32, 1)
    index, weight = gn.route(logits, 4)
    for call in (lambda: gn.route(logits, 0), lambda: gn.route(logits, 17), lambda: gn.route(logits, 4, "tanh"), lambda: gn.route(logits[0], 4),
                 lambda: gn.route(logits, 4, bias=torch.zeros(15, device="cuda")), lambda: gn.route_grad(weight[:, :3], logits, index),
                 lambda: gn.route_grad(weight, logits, index[:4])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gn.route(logits.double(), 4), lambda: gn.route(logits, 4, bias=torch.zeros(16, device="cuda", dtype=torch.float16)),
                 lambda: gn.route_grad(weight, logits, index.long()), lambda: gn.route_grad(weight.half(), logits, index), lambda: gn.route(logits, 4.0)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: gn.route(logits, 4, groups=3), lambda: gn.route(logits, 4, groups=8, top_groups=1), lambda: gn.route(logits, 4, groups=4, top_groups=5),
                 lambda: gn.route(logits, 4, group_best=3), lambda: gn.route(logits, 4, scale=math.inf)):
        with pytest.raises(gn.GnError):
            call()


def test_a_scale_is_a_number():
    logits = rand((4, 16), torch.float32, 1)
    assert torch.equal(gn.route(logits, 2, scale=2)[1], gn.route(logits, 2, scale=2.0)[1])
    for bad in ("1", None, True, torch.ones(1), 1j):
        with pytest.raises(TypeError, match="scale"):
            gn.route(logits, 2, scale=bad)
    for bad in (10 ** 400, -1e301, math.nan, math.inf):
        with pytest.raises(gn.GnError, match="scale"):
            gn.route(logits, 2, scale=bad)
