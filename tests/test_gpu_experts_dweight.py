"""The gradient of the routing weights, an FP32 result of 16-bit operands, is as near to its formula as FP32 sums are, for any length of them."""
import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import act64, rand
from mixture_common import choices, used, weights_of

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def dweight64(dy, index, gate, up, w_down, act):
    out = torch.zeros(index.shape, dtype=torch.float64, device="cuda")
    for e, t, j in used(index, w_down.shape[0]):
        pair = t * index.shape[1] + j
        out[t, j] = ((dy[t].double() @ w_down[e].double()) * act64(act, gate[pair].double())[0] * up[pair].double()).sum(1)
    return out


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("tokens,cols,inner,experts,k", [(600, 2048, 512, 4, 2), (300, 4096, 328, 3, 1), (100, 16384, 264, 2, 1), (257, 1000, 1001, 4, 2), (40, 3001, 77, 8, 3), (900, 520, 256, 2, 2)])
def test_dweight_is_not_cut_off(t, act, tokens, cols, inner, experts, k):
    """In the 2-norm over all pairs.  q = sum over `cols` terms is made of sums of at most 512, in 32 additions of 16 products, each of which cuts off at most 2^-23 of a sum (2^-24 on average, the same way): 32 2^-24
    = 1.9e-6 of a sum that had its last size all the time.  These are sums of random signs, whose size grows with the root of the terms, and what is cut off is in the direction of the sum then, not of
    the last one, so a third of it at most is left: 0.64e-6.  FP32 additions of up to 32 such sums, the 16-bit activation (silu: ex2 and rcp off by up to (4 + |v|) 2^-23, random from element to element) and
    the sum over `inner` add 0.1e-6: 1e-6 in all.  Sums of 2048 terms and more that stay in the tensor core are 2e-6 off and more."""
    t = TYPES[t]
    x = rand((tokens, cols), t, 1)
    index, weight = choices(tokens, experts, k)
    w = weights_of(experts, cols, inner, t)
    _, gate, up = gn.experts(x, index, weight, *w, act, save=True)
    dy = rand(x.shape, t, 9, 0.3)
    got = gn.experts_grad(dy, x, index, weight, gate, up, *w, act)[1]
    want = dweight64(dy, index, gate, up, w[2], act)
    off = float((got.double() - want).norm() / want.norm())
    assert off < 1e-6, off
