"""Dropout from the counter-based generator: masks word for word, values, layouts, gradients."""
import ctypes as C

import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import E, TYPES, mask_of, philox_words, rand, tiny, u, within

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 3), (3, 1), (5, 2), (7, 5), (131, 617), (64, 8), (33, 130), (1, 100003), (300, 1024), (2, 16), (17, 4100)]


def test_words_of_the_generator():
    """Known answer of Philox4x32-10 for the zero counter and key (published with the method)."""
    assert [hex(int(w)) for w in philox_words(4, 0, 0)] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]




@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("t", TYPES)
def test_values(t, shape, p, residual):
    t, key, step = TYPES[t], 0xDEADBEEF12345678, 0x1000000005
    x, r = rand(shape, t, 1, 1.0, 3.0), rand(shape, t, 2) if residual else None
    y = gn.dropout(x, p, key, step, residual=r)
    keep = mask_of(shape, p, key, step)
    kept = torch.where(keep, x.double() / max(1 - p, 1e-300), 0.0)
    ref = kept + (r.double() if residual else 0.0)
    # the scale rounded to FP32, the product, the sum, and the rounding to the type
    within(y, ref, u(t) * ref.abs() + tiny(t) + 3 * E * kept.abs() + E * ref.abs(), "y")
    if not residual:
        assert bool((y[~keep] == 0).all())


@pytest.mark.parametrize("pads", [(1, 0), (3, 8), (8, 3), (0, 5)])
@pytest.mark.parametrize("t", TYPES)
def test_the_mask_goes_by_the_element_and_not_by_its_place(t, pads):
    t = TYPES[t]
    x, r = rand((70, 129), t, 1, pad=pads[0]), rand((70, 129), t, 2, pad=pads[1])
    assert torch.equal(gn.dropout(x, 0.3, 5, 6, residual=r), gn.dropout(x.contiguous(), 0.3, 5, 6, residual=r.contiguous()))


@pytest.mark.parametrize("offset", range(1, 8))
def test_misaligned_bases(offset):
    flat = rand((1, 64 * 1024 + 8), torch.bfloat16, 4)[0]
    x = flat[offset: offset + 64 * 1024].view(64, 1024)
    assert torch.equal(gn.dropout(x, 0.3, 5), gn.dropout(x.clone(), 0.3, 5))


def test_types_draw_the_same_mask_and_keys_and_steps_another():
    one = lambda t, key, step: gn.dropout(torch.ones(100, 333, dtype=t, device="cuda"), 0.5, key, step) != 0
    base = one(torch.float32, 11, 12)
    assert torch.equal(base, one(torch.bfloat16, 11, 12)) and torch.equal(base, one(torch.float16, 11, 12))
    for key, step in ((12, 12), (11, 13), (11 + (1 << 32), 12), (11, 12 + (1 << 32))):
        share = float((one(torch.float32, key, step) == base).double().mean())
        assert abs(share - 0.5) < 7 * 0.5 / 33300 ** 0.5


def test_nothing_of_a_dropped_element_is_left():
    x = torch.full((50, 70), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[::2] = float("inf")
    keep, y = mask_of((50, 70), 0.4, 1, 2), gn.dropout(x, 0.4, 1, 2)
    assert bool((y[~keep] == 0).all()) and not bool(y[keep].isfinite().any())
    assert bool((gn.dropout(x, 1.0, 1, 2) == 0).all())


def test_step_from_the_device_and_replays():
    x = rand((65, 130), torch.float16, 1)
    step = torch.tensor([3], dtype=torch.int64, device="cuda")
    assert torch.equal(gn.dropout(x, 0.2, 9, 4, device_step=step), gn.dropout(x, 0.2, 9, 7))
    assert torch.equal(gn.dropout(x, 0.2, 9, 2 ** 64 - 1, device_step=step), gn.dropout(x, 0.2, 9, 2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = gn.dropout(x, 0.2, 9, 4, device_step=step)
        step += 1
    for k in range(3):
        graph.replay()
        assert torch.equal(y, gn.dropout(x, 0.2, 9, 7 + k))


def test_the_backward_pass_is_the_call_itself():
    """<dropout(x), c> = <x, dropout(c)>: the map is linear with a diagonal matrix."""
    x, c = rand((90, 33), torch.float32, 1), rand((90, 33), torch.float32, 2)
    a = (gn.dropout(x, 0.25, 3, 4).double() * c.double()).sum()
    b = (x.double() * gn.dropout(c, 0.25, 3, 4).double()).sum()
    assert abs(float(a - b)) < 4 * E * float((x.double() * c.double()).abs().sum()) * 4 / 3


@pytest.mark.parametrize("ld", [40, 41, 48])
def test_in_place_and_what_is_left_alone(ld):
    rows, cols, err = 11, 40 if ld != 41 else 39, C.create_string_buffer(200)
    x, r = rand((rows, cols), torch.float16, 1), rand((rows, cols), torch.float16, 2)
    want = gn.dropout(x, 0.5, 1, 2, residual=r)
    for place in range(2):
        b = []
        for m in (x, r):
            w = torch.full((rows + 2, ld), 7.0, dtype=torch.float16, device="cuda")
            w[:rows, :cols] = m
            b.append(w)
        assert gn.lib().gn_dropout(2, rows, cols, b[0].data_ptr(), ld, b[1].data_ptr(), ld, b[place].data_ptr(), ld, 0.5, 1, 2, None,
                                   torch.cuda.current_stream().cuda_stream, err, 200) == 0, err.value
        assert torch.equal(b[place][:rows, :cols], want)
        assert bool((b[place][rows:] == 7).all()) and bool((b[place][:, cols:] == 7).all())


def test_no_rows_and_refusals():
    assert gn.dropout(torch.empty(0, 5, device="cuda"), 0.1, 1).shape == (0, 5)
    x = rand((4, 16), torch.bfloat16, 1)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(gn.GnError, match="p must"):
            gn.dropout(x, p, 1)
    for bad in (lambda: gn.dropout(x.double(), 0.1, 1), lambda: gn.dropout(x, 0.1, 1, residual=x.float()),
                lambda: gn.dropout(x, 0.1, 1, device_step=torch.zeros(1, dtype=torch.int32, device="cuda")),
                lambda: gn.dropout(x, 0.1, 1, device_step=torch.zeros(1, dtype=torch.int64))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: gn.dropout(x, 0.1, 1, residual=x[:2]), lambda: gn.dropout(x.T, 0.1, 1),
                lambda: gn.dropout(x, 0.1, 1, device_step=torch.zeros(2, dtype=torch.int64, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
