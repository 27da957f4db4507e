"""The choice of groups by sums of values that are large beside their scores, against sums of scores and of biases in 64 bits."""
import math

import pytest
import torch

from feedforward_common import rand
from test_gpu_route import check

pytestmark = pytest.mark.gpu
INF = math.inf


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups", [(16, 4), (256, 8), (60, 6), (1024, 32)])
@pytest.mark.parametrize("size", [64.0, 4096.0, 1e6])
def test_group_sums_of_biases_that_cancel(score, experts, groups, size):
    """Two best values of a group that are large and of opposite signs: their sum is that of the scores, of which FP32 has lost the last digits, or all."""
    logits = rand((1500, experts), torch.float32, experts, 1.5)
    bias = torch.full((experts,), -size, device="cuda")
    bias[:: experts // groups] = size
    for top in (1, groups // 2, groups - 1):
        check(logits, 2, score, bias, groups, top, 2)
    bias[-(experts // groups):] = -INF                       # (and a group that is kept out)
    check(logits, 2, score, bias, groups, groups // 2, 2)


def test_group_sums_beyond_fp32():
    """Sums of two biases near the largest number: finite, and in their order."""
    logits = rand((20, 16), torch.float32, 1)
    for sign in (1.0, -1.0):
        bias = sign * torch.tensor([3.0e38, 3.1e38, 3.3e38, 3.2e38], device="cuda").repeat_interleave(4)
        for top in (1, 2, 3):
            check(logits, 2, "sigmoid", bias, 4, top, 2)
