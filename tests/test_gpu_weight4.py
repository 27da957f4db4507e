"""4-bit weights: their layout, and products with them against a plain form in 64 bits."""
import math

import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import E, TYPES, act64, product, rand, tiny, u, within
from mixture_common import ACT, check_experts, choices

pytestmark = pytest.mark.gpu

ACTS = ["sigmoid", "silu", "gelu", "gelu_tanh", "relu"]


def quarters(shape, group, t, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q = torch.randint(0, 16, shape, generator=g, device="cuda", dtype=torch.uint8)
    scale = (0.5 + torch.rand((*shape[:-1], -(-shape[-1] // group)), generator=g, device="cuda")) * 0.25 * shape[-1] ** -0.5
    return q, scale.to(t)


def values(q, scale, group):
    return (q.double() - 8) * scale.double().repeat_interleave(group, -1)[..., : q.shape[-1]]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("shape", [(1, 1), (16, 128), (17, 129), (5, 40), (100, 321), (3, 20, 70), (2, 33, 256)])
def test_layout(t, group, shape):
    q, scale = quarters(shape, group, TYPES[t], 1)
    w = gn.pack4(q, scale, group)
    experts, rows, cols = (1, *shape)[-3:]
    assert w.shape == shape and w.q.numel() == experts * -(-rows // 16) * -(-cols // 128) * 1024
    # the documented places
    e, r, c = torch.meshgrid(*(torch.arange(n, device="cuda") for n in (experts, rows, cols)), indexing="ij")
    word = ((e * -(-rows // 16) + r // 16) * -(-cols // 128) + c // 128) * 256 + r % 16 // 8 * 128 + r % 8 * 16 + c // 8 % 4 * 4 + c % 128 // 32
    got = w.q.view(torch.int32)[word] >> (4 * (c % 8 // 2) + 16 * (c % 2)) & 15
    assert torch.equal(got.view(shape).to(torch.uint8), q)
    each = 128 // group
    at = (((e * -(-rows // 16) + r // 16) * -(-cols // 128) + c // 128) * 16 + r % 16) * each + c % 128 // group
    assert torch.equal(w.scale[at].view(shape), scale.repeat_interleave(group, -1)[..., :cols])
    kept = torch.zeros_like(w.scale, dtype=torch.bool)
    kept[at] = True
    assert bool((w.scale[~kept] == 0).all())
    nibbles = torch.stack([w.q & 15, w.q >> 4], 1)
    assert int((nibbles != 8).sum()) == int((q != 8).sum())
    assert torch.equal(gn.unpack4(w), values(q, scale, group).to(TYPES[t]))
    wide = torch.full((*shape[:-1], cols + 3), 255, device="cuda", dtype=torch.uint8)
    wide[..., :cols] = q + 16 * 5                            # (the upper four bits do not count)
    again = gn.pack4(wide[..., :cols], scale, group)
    assert torch.equal(again.q, w.q) and torch.equal(again.scale, w.scale)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantize(t, group):
    w = rand((70, 300), TYPES[t], 1, 0.1, pad=2)
    w[3, :128] = 0
    w[5, 7] = 9.0
    got = gn.unpack4(gn.quantize4(w, group)).double()
    n = -(-300 // group)
    wide = torch.zeros(70, n * group, device="cuda", dtype=torch.float32)
    wide[:, :300] = w.float()
    most = wide.view(70, n, group).abs().amax(2)
    s = (most.double() / 7).float().to(TYPES[t]).float()[:, :, None]       # (FP32 by a number is multiplied with its reciprocal there)
    q = torch.where(s == 0, 0.0, torch.round(wide.view(70, n, group) / s).clamp(-8, 7))
    assert torch.equal(got, (q * s).view(70, -1)[:, :300].to(TYPES[t]).double())
    both = gn.quantize4(torch.stack([w, w]), group)
    assert both.shape == (2, 70, 300) and torch.equal(gn.unpack4(both)[1].double(), got)
    w[9, 11], w[10, 12] = math.nan, math.inf
    bad = gn.unpack4(gn.quantize4(w, group))
    assert bool(bad[9, :group].isnan().all()) and bool(bad[10, :group].isnan().all()) and bool(bad[11].isfinite().all())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens,rows,cols", [(1, 1, 1), (1, 16, 128), (2, 17, 129), (7, 40, 1000), (8, 500, 256), (9, 33, 513), (31, 100, 65), (33, 64, 300), (70, 257, 640), (1, 1000, 4096),
                                              (3, 4099, 200), (5, 128, 9000)])
def test_matvec(t, group, tokens, rows, cols):
    q, scale = quarters((rows, cols), group, TYPES[t], tokens)
    w = gn.pack4(q, scale, group)
    for pad in (0, 3):
        x = rand((tokens, cols), TYPES[t], 2, pad=pad)
        ref, err = product(x.double(), values(q, scale, group), 0, 0)
        within(gn.matvec4(x, w), ref, err + u(TYPES[t]) * ref.abs() + tiny(TYPES[t]), "y")


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens,cols,inner", [(1, 1, 1), (1, 128, 16), (2, 129, 17), (8, 1000, 300), (9, 33, 513), (40, 264, 136), (1, 2048, 1024)])
def test_layer(t, group, tokens, cols, inner):
    x = rand((tokens, cols), TYPES[t], 2, pad=3)
    parts = [quarters(s, group, TYPES[t], 3 + i) for i, s in enumerate(((inner, cols), (inner, cols), (cols, inner)))]
    w = [gn.pack4(*p, group) for p in parts]
    act = ACTS[(tokens + cols + inner) % 5]
    one = torch.zeros(tokens, 1, dtype=torch.int32, device="cuda")
    check_experts(gn.gated_ffn4(x, *w, act), x, one, torch.ones(tokens, 1, device="cuda"), [values(*p, group)[None] for p in parts], act, TYPES[t], row=0.0,
                  h_round=0.0 if t == "f32" else 2.0 ** -17 / u(TYPES[t]))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("tokens,cols,inner,experts,k", [(1, 128, 16, 1, 1), (1, 200, 72, 64, 8), (8, 264, 136, 16, 4), (50, 72, 40, 3, 2), (200, 129, 65, 4, 2), (33, 64, 64, 300, 6), (2000, 40, 24, 5, 1)])
def test_experts(t, group, tokens, cols, inner, experts, k):
    x = rand((tokens, cols), TYPES[t], 2)
    index, weight = choices(tokens, experts, k)
    parts = [quarters((experts, *s), group, TYPES[t], 3 + i) for i, s in enumerate(((inner, cols), (inner, cols), (cols, inner)))]
    w = [gn.pack4(*p, group) for p in parts]
    act = ACTS[(tokens + cols + inner) % 5]
    plain = [values(*p, group) for p in parts]
    doubtful = index.clone()
    doubtful[::3, 0] = -1
    doubtful[1::4] = experts
    for table in (index, doubtful, torch.zeros_like(index)):
        got = gn.gated_ffn4(x, *w, act, index=table, weight=weight)
        check_experts(got, x, table, weight, plain, act, TYPES[t], row=0.0, h_round=0.0 if t == "f32" else 2.0 ** -17 / u(TYPES[t]))
        assert bool((got[((table < 0) | (table >= experts)).all(1)] == 0).all())


def test_large_and_infinite_tokens_in_fp32():
    """The three parts of an FP32 number: none of them overflows, and an infinity stays one."""
    q, scale = torch.full((16, 128), 9, device="cuda", dtype=torch.uint8), torch.ones(16, 1, device="cuda")
    w = gn.pack4(q, scale)
    x = torch.zeros(4, 128, device="cuda")
    x[0, 5], x[1, 5], x[2, 5], x[3, 5] = 3.4028234e38, 1.1754944e-38, math.inf, math.nan
    y = gn.matvec4(x, w)
    assert bool((y[0] == x[0, 5]).all()) and bool((y[1] == x[1, 5]).all()) and bool((y[2] == math.inf).all()) and bool(y[3].isnan().all())


@pytest.mark.parametrize("t", TYPES)
def test_streams_and_graphs(t):
    x, (index, weight) = rand((9, 136), TYPES[t], 2), choices(9, 6, 2)
    w = [gn.pack4(*quarters((6, *s), 64, TYPES[t], i), 64) for i, s in enumerate(((72, 136), (72, 136), (136, 72)))]
    flat = gn.pack4(*quarters((200, 136), 64, TYPES[t], 9), 64)
    every = lambda stream=None: (gn.matvec4(x, flat, stream=stream), gn.gated_ffn4(x, *w, index=index, weight=weight, stream=stream))
    first = every()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other, again = every(side), every()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(first, other, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = every()
    x.copy_(rand(x.shape, TYPES[t], 77))
    index.copy_(choices(9, 6, 2, 5)[0])
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, every()))
    none = gn.gated_ffn4(x[:0], *w, index=index[:0], weight=weight[:0])
    assert none.shape == (0, 136) and gn.matvec4(x[:0], flat).shape == (0, 200)


def test_refusals():
    t = torch.bfloat16
    x = rand((4, 64), t, 1)
    q, scale = quarters((32, 64), 32, t, 1)
    w, down = gn.pack4(q, scale, 32), gn.pack4(*quarters((64, 32), 32, t, 2), 32)
    index, weight = choices(4, 3, 2)
    many = gn.pack4(*quarters((3, 32, 64), 32, t, 1), 32)
    for call in (lambda: gn.pack4(q, scale, 64), lambda: gn.pack4(q, scale, 48), lambda: gn.pack4(q[0], scale[0], 32), lambda: gn.pack4(q, scale[:31], 32), lambda: gn.pack4(q.t(), scale, 32),
                 lambda: gn.matvec4(x[:, :63], w), lambda: gn.matvec4(x, many), lambda: gn.gated_ffn4(x, w, w, w), lambda: gn.gated_ffn4(x, w, w, down, index=index, weight=weight),
                 lambda: gn.gated_ffn4(x, w, w, down, "tanh"), lambda: gn.gated_ffn4(x, w, w, gn.quantize4(rand((64, 32), t, 1), 64)), lambda: gn.quantize4(x, 16)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gn.pack4(q.int(), scale, 32), lambda: gn.pack4(q, scale.double(), 32), lambda: gn.matvec4(x.float(), w), lambda: gn.matvec4(x, q), lambda: gn.gated_ffn4(x, q, q, q),
                 lambda: gn.quantize4(x.double()), lambda: gn.quantize4(x.cpu()), lambda: gn.unpack4(x)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("inner", [1, 17, 64])
def test_infinite_tokens_through_a_layer(t, inner):
    """Positive weights alone, so that no infinity meets a zero or its opposite: the result is infinite too, whatever is past the last hidden unit."""
    t = TYPES[t]
    ones = lambda *shape: gn.pack4(torch.full(shape, 9, device="cuda", dtype=torch.uint8), torch.ones(*shape[:-1], -(-shape[-1] // 64), device="cuda", dtype=t), 64)
    x = torch.full((3, 40), 0.25, device="cuda", dtype=t)
    x[1, 7] = math.inf
    y = gn.gated_ffn4(x, ones(inner, 40), ones(inner, 40), ones(40, inner), "relu")
    assert bool((y[1] == math.inf).all()) and bool((y[::2] == torch.tensor(100.0 * inner, dtype=t)).all())
    index, weight = torch.tensor([[0], [1], [1]], device="cuda", dtype=torch.int32), torch.ones(3, 1, device="cuda")
    y = gn.gated_ffn4(x, ones(2, inner, 40), ones(2, inner, 40), ones(2, 40, inner), "relu", index, weight)
    assert bool((y[1] == math.inf).all()) and bool(y[::2].isfinite().all())


@pytest.mark.parametrize("t", TYPES)
def test_the_most_tokens(t):
    t, n = TYPES[t], (1 << 19) - 1
    q, scale = quarters((24, 40), 32, t, 1)
    x = rand((n, 40), t, 2)
    ref, err = product(x.double(), values(q, scale, 32), 0, 0)
    within(gn.matvec4(x, gn.pack4(q, scale, 32)), ref, err + u(t) * ref.abs() + tiny(t), "y")
    # (one record a row, so that every token's sums have one order in any call)
    w = [gn.pack4(*quarters(s, 32, t, 3), 32) for s in ((17, 40), (17, 40), (40, 17))]
    y = gn.gated_ffn4(x, *w)
    for part in (slice(0, 50), slice(n // 2, n // 2 + 50), slice(n - 50, n)):
        assert torch.equal(y[part], gn.gated_ffn4(x[part], *w))
    w, (index, weight) = [gn.pack4(*quarters((3, *s), 32, t, 3), 32) for s in ((17, 40), (17, 40), (40, 17))], choices(n // 2, 3, 2)
    y = gn.gated_ffn4(x[: n // 2], *w, index=index, weight=weight)
    for part in (slice(0, 50), slice(n // 2 - 50, n // 2)):
        assert torch.equal(y[part], gn.gated_ffn4(x[part], *w, index=index[part], weight=weight[part]))
