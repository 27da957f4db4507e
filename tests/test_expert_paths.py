"""The sizes by which the GPU tests reach each FP32 form of a mixture's experts do reach it."""
import pytest

from expert_paths import BACKWARD, FORWARD, path


@pytest.mark.parametrize("name,shape", [(n, s) for n in FORWARD for s in FORWARD[n]])
def test_forward(name, shape):
    assert path(*shape, False) == name


@pytest.mark.parametrize("name,shape", [(n, s) for n in BACKWARD for s in BACKWARD[n]])
def test_backward(name, shape):
    assert path(*shape, True) == name
