"""Routing weights whose scores are far from one another or far from one, and their gradients, against shares formed from logarithms in 64 bits."""
import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import TYPES, rand

pytestmark = pytest.mark.gpu


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
