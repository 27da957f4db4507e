"""FP32 numbers in three BF16 parts, as a mixture's experts multiply them on the tensor cores."""
import math

import pytest
import torch

import paper_1802_00130_b200 as gn
from expert_paths import path

pytestmark = pytest.mark.gpu

SHAPE = (700, 200, 333, 6, 3)
LARGEST = torch.finfo(torch.float32).max


def one_term_each(value):
    """Tokens of a single element, so that a projection is one product; (x, that element's column)."""
    tokens, cols = SHAPE[:2]
    at = torch.arange(tokens, device="cuda") % cols
    return torch.zeros(tokens, cols, device="cuda").scatter_(1, at[:, None], value[:, None]), at


def gate_of(x, w_gate):
    tokens, cols, inner, experts, k = SHAPE
    assert path(*SHAPE, False) == "tensor"
    index = (torch.arange(tokens * k, device="cuda") % experts).to(torch.int32).view(tokens, k)
    w_up, w_down = torch.ones(experts, inner, cols, device="cuda"), torch.ones(experts, cols, inner, device="cuda")
    _, gate, _ = gn.experts(x, index, torch.ones(tokens, k, device="cuda"), w_gate, w_up, w_down, save=True)
    return gate.view(tokens, k, inner), index.long()


def numbers(n, seed, awkward):
    """Numbers of either sign whose later parts are as large as they can be, or any."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    size = torch.exp2(torch.randint(-8, 9, (n,), generator=g, device="cuda").float())
    sign = 1 - 2 * torch.randint(0, 2, (n,), generator=g, device="cuda").float()
    if not awkward:
        return (1 + torch.rand(n, generator=g, device="cuda")) * size * sign
    near = torch.tensor([1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -8 + 2.0 ** -16 - 2.0 ** -23, 1 + 2.0 ** -8 - 2.0 ** -23, 1 + 2.0 ** -7 - 2.0 ** -15 + 2.0 ** -16], device="cuda")
    return near[torch.randint(0, 4, (n,), generator=g, device="cuda")] * size * sign


@pytest.mark.parametrize("awkward", [True, False])
def test_a_product_leaves_out_less_than_2_to_the_minus_23(awkward):
    """What is left out of a b: a_1 b_2, a_2 b_1 and a_2 b_2.  Parts are rounded to nearest, so |a_1| <= 2^-8 2^e and |a_2| <= 2^-16 2^e where 2^e <= |a|: (2 2^-24 + 2^-32) |a b|.
    The six other products are added with at most one step of the result, 2^-23 of it, in the last addition, and steps of sums that are 2^-7 of it at most in the five before."""
    tokens, cols, inner, experts, k = SHAPE
    a, b = numbers(tokens, 1, awkward), numbers(experts * inner * cols, 2, awkward).view(experts, inner, cols)
    x, at = one_term_each(a)
    gate, index = gate_of(x, b)
    want = a.double()[:, None, None] * b.double()[index, :, at[:, None]]
    assert float(((gate.double() - want) / want).abs().max()) <= 2.0 ** -23 * (1 + 2.0 ** -8 + 1 + 5 * 2.0 ** -7)


def test_largest_numbers_infinities_and_nan():
    """The leading part of a number near the largest is not rounded to infinity; an infinite or undefined element leaves nothing finite of what it meets, and nothing else is touched by it."""
    tokens, cols, inner, experts, k = SHAPE
    a = torch.full((tokens,), LARGEST, device="cuda")
    a[1::7] = -LARGEST
    a[2::7] = LARGEST * (1 - 2.0 ** -9)
    a[3::7] = LARGEST * (1 - 2.0 ** -8)
    b = numbers(experts * inner * cols, 2, False).view(experts, inner, cols) * 2.0 ** -30
    x, at = one_term_each(a)
    gate, index = gate_of(x, b)
    want = a.double()[:, None, None] * b.double()[index, :, at[:, None]]
    assert float(((gate.double() - want) / want).abs().max()) <= 2.0 ** -23 * 2.1
    quiet = torch.tensor([0x7FC00000, 0x7F800001, -1, 0x7FFFFFFF, -0x7FFFFF], dtype=torch.int32, device="cuda").view(torch.float32)     # (NaN of several patterns)
    for value in (math.inf, -math.inf, *quiet.split(1)):
        bad = x.clone()
        bad[5, at[5]] = value
        other, _ = gate_of(bad, b)
        assert not bool(other[5].isfinite().any())
        other[5] = gate[5]
        assert torch.equal(other, gate)


@pytest.mark.parametrize("shape", [SHAPE, (300, 264, 136, 6, 2)])
def test_infinities_are_those_of_the_formula(shape):
    """An infinite token or weight: infinite projections of the formula's signs, NaN where it meets a zero, and the same on FMAs (the second shape) and on the tensor cores."""
    tokens, cols, inner, experts, k = shape
    assert path(*shape, False) == ("tensor" if shape == SHAPE else "small")
    x, w_gate = numbers(tokens * cols, 1, True).view(tokens, cols).clone(), numbers(experts * inner * cols, 2, True).view(experts, inner, cols).clone()
    w_up, w_down = w_gate.flip(1).clone(), torch.ones(experts, cols, inner, device="cuda")
    x[5, 7], x[6, 9], x[8, cols - 1] = math.inf, -math.inf, math.inf
    x[10, 3] = 0
    w_gate[1, 4, 3] = math.inf
    w_gate[2, 5, 7] = 0
    w_up[0, 2, 11] = -math.inf
    index = (torch.arange(tokens * k, device="cuda") % experts).to(torch.int32).view(tokens, k)
    y, gate, up = gn.experts(x, index, torch.ones(tokens, k, device="cuda"), w_gate, w_up, w_down, "relu", save=True)
    for got, w in ((gate, w_gate), (up, w_up)):
        # (term by term, so that the 64-bit form meets infinities as the formula has them)
        want = torch.stack([(x.double()[:, None, :] * w[e].double()[None]).sum(2) for e in range(experts)], 1).gather(1, index.long()[:, :, None].expand(-1, -1, inner))
        got = got.view(tokens, k, inner)
        assert bool(want.isinf().any()) and bool(want.isnan().any() or w is w_up)
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
        assert torch.equal(got[want.isinf()].double(), want[want.isinf()])
