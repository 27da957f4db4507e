"""Routing weights whose scores are far from one another or far from one, and their gradients, against shares formed from logarithms in 64 bits."""
import math

import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import E, TYPES, rand, tiny, u, within

pytestmark = pytest.mark.gpu
INF = math.inf


def shares64(logits, index, score):
    """Scores of the chosen over their sum: exp(log s_j - the largest - log of the sum), for which no score is too small.  Zero where none of them has one: with
    softmax of -inf alone, with sigmoid where all are below exp(-700), which 64 bits cannot hold either."""
    z = logits.double().gather(1, index.long())
    log = -torch.nn.functional.softplus(-z) if score == "sigmoid" else z
    log = torch.where(z == -INF, -INF, log)
    top = log.amax(1, keepdim=True)
    if score == "sigmoid":
        log = torch.where(top < -700, -INF, log)
        top = log.amax(1, keepdim=True)
    e = (log - top.masked_fill(top == -INF, 0)).exp()
    total = e.sum(1, keepdim=True)
    return e / total.masked_fill(total == 0, 1)


# A share exp(z - m) / sum: z - m is rounded (its distance, below 100 where the share is above FP32's smallest, in steps of E of the share), the exponential 4 E, 1 + exp(z) and
# the quotient 6 E, the sum of up to 32 of them 32 + 100 E, the division and the scale 4 E.
SHARE = 250 * E


def chosen_by_bias(experts, picked):
    """A bias that makes the choice, whatever the scores are: the picked experts in their order."""
    bias = torch.full((experts,), -10.0, device="cuda")
    for i, e in enumerate(picked):
        bias[e] = 100.0 - 2 * i
    return bias


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("experts,k", [(3, 2), (40, 5), (256, 8), (1000, 32)])
@pytest.mark.parametrize("below", [3.0, 60.0, 88.0, 95.0, 104.0, 200.0, 30000.0])
def test_shares_of_experts_far_below_the_rows_largest(t, experts, k, below):
    """A bias chooses experts whose softmax scores are tiny beside that of another: their shares still add up to the scale."""
    logits = rand((50, experts), TYPES[t], experts, 1.5)
    logits -= below
    logits[:, 0] = 0
    picked = list(range(experts - 1, experts - 1 - k, -1))
    index, weight = gn.route(logits, k, "softmax", chosen_by_bias(experts, picked), renormalise=True, scale=2.5)
    assert index.tolist() == [picked] * 50
    want = 2.5 * shares64(logits, index, "softmax")
    within(weight, want, want * SHARE + 1e-37, "weight")
    dweight = rand((50, k), torch.float32, 2)
    got = gn.route_grad(dweight, logits, index, "softmax", True, 2.5)
    check_gradient(got, dweight, logits, index, "softmax", 2.5)


def check_gradient(got, dweight, logits, index, score, scale):
    """p_j (u_j - sum u p), and with sigmoid times 1 - s_j: sums of k terms, each with the share's error twice and k + 8 roundings."""
    p, uj = shares64(logits, index, score), dweight.double() * scale
    d = p * (uj - (uj * p).sum(1, keepdim=True))
    if score == "sigmoid":
        d = d * torch.sigmoid(-logits.double().gather(1, index.long()))
    ref = torch.zeros(logits.shape, dtype=torch.float64, device="cuda").scatter_add_(1, index.long(), d)
    bound = torch.zeros_like(ref).scatter_add_(1, index.long(), p * uj.abs().amax(1, keepdim=True)) * 2 * (2 * SHARE + (index.shape[1] + 8) * E)
    within(got, ref, bound + ref.abs() * u(logits.dtype) + tiny(logits.dtype) + 1e-37, "dlogits")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("experts,k", [(2, 2), (40, 5), (256, 8), (1000, 32)])
@pytest.mark.parametrize("middle", [80.0, 0.0, -40.0, -80.0, -86.0, -90.0, -100.0, -300.0, -600.0, -30000.0])
@pytest.mark.parametrize("spread", [1.5, 15.0])
def test_shares_of_sigmoids_far_from_one(t, experts, k, middle, spread):
    """Scores below FP32's smallest number still have shares."""
    logits = rand((50, experts), TYPES[t], experts, spread, middle)
    index, weight = gn.route(logits, k, "sigmoid", renormalise=True, scale=1.5)
    assert torch.equal(index.long(), logits.double().sort(dim=1, descending=True, stable=True).indices[:, :k])
    want = 1.5 * shares64(logits, index, "sigmoid")
    within(weight, want, want * SHARE + 1e-37, "weight")
    dweight = rand((50, k), torch.float32, 2)
    check_gradient(gn.route_grad(dweight, logits, index, "sigmoid", True, 1.5), dweight, logits, index, "sigmoid", 1.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_some_of_the_chosen_are_masked(score):
    """A bias takes experts with logits of -inf: they have the share 0, and where there is nothing else so have all."""
    logits = torch.full((4, 24), -120.0, device="cuda")
    logits[:, 0] = 3.0
    logits[0, 20:] = -INF
    logits[1, 21] = -INF
    logits[2, 20], logits[2, 21:] = -INF, torch.finfo(torch.float32).min
    index, weight = gn.route(logits, 4, score, chosen_by_bias(24, [20, 21, 22, 23]), renormalise=True)
    assert index.tolist() == [[20, 21, 22, 23]] * 4
    want = shares64(logits, index, score)
    within(weight, want, want * SHARE, "weight")
    assert weight[0].tolist() == [0.0] * 4 and weight[1, 1] == 0 and weight[2, 0] == 0
    dweight = rand((4, 4), torch.float32, 2)
    check_gradient(gn.route_grad(dweight, logits, index, score, True), dweight, logits, index, score, 1.0)


@pytest.mark.parametrize("bias", [False, True])
def test_a_row_with_a_nan_or_an_infinity_has_no_shares(bias):
    """With softmax, whether or not it is among the chosen, which are the first ones then."""
    logits = rand((4, 40), torch.float32, 1)
    logits[0, 30] = math.nan
    logits[1, 30] = INF
    logits[2, 1] = INF
    b = torch.zeros(40, device="cuda") if bias else None
    for renormalise in (False, True):
        index, weight = gn.route(logits, 4, "softmax", b, renormalise=renormalise)
        assert bool(weight[:3].isnan().all()) and bool(weight[3].isfinite().all())
    weight = gn.route(logits, 4, "sigmoid", b, renormalise=True)[1]
    assert bool(weight.isfinite().all())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,experts", [(1, 1), (1, 2), (77, 60), (4001, 256), (5, 1024)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_one_weight_over_itself_has_no_gradient(t, tokens, experts, score):
    """One choice with renormalise: w = scale for any logits, so the gradient is zero, and no rounding may leave anything."""
    logits = rand((tokens, experts), TYPES[t], 3, 1.5)
    index, weight = gn.route(logits, 1, score, renormalise=True, scale=2.5)
    assert bool((weight == 2.5).all())
    got = gn.route_grad(rand((tokens, 1), torch.float32, 4), logits, index, score, True, 2.5)
    assert bool((got == 0).all())
