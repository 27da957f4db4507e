"""The calls of a mixture of experts take as many pairs of token and choice as they say, for a number of choices that does not divide the limit too."""
import pytest

import paper_1802_00130_b200 as gn
from test_experts_args import ffn4, mixture


@pytest.mark.parametrize("k", [1, 2, 3, 5, 7, 31, 32])
@pytest.mark.parametrize("type", [0, 1, 2])
def test_pairs_below_the_limit(type, k):
    lib = gn.lib()
    most = -(-(1 << 28) // k) - 1              # the last number of tokens with tokens k < 2^28
    for backward in (0, 1):
        assert lib.gn_experts_workspace(mixture(type=type, k=k, tokens=most), backward) > 0 and lib.gn_experts_workspace(mixture(type=type, k=k, tokens=most + 1), backward) < 0
        assert lib.gn_experts_workspace(mixture(type=type, k=k, tokens=1 << 62), backward) < 0
    most = -(-(1 << 19) // k) - 1
    assert lib.gn_gated_ffn4_workspace(ffn4(type=type, k=k, tokens=most)) > 0 and lib.gn_gated_ffn4_workspace(ffn4(type=type, k=k, tokens=most + 1)) < 0
    assert lib.gn_gated_ffn4_workspace(ffn4(type=type, k=k, tokens=1 << 62)) < 0
