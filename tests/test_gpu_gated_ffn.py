"""Gated feed-forward block and its backward pass against a plain form in 64 bits."""
import ctypes as C
import math

import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import E, TYPES, act64, product, rand, tiny, u, within

pytestmark = pytest.mark.gpu

ACTS = ["sigmoid", "silu", "gelu", "gelu_tanh", "relu"]
# rows, cols, inner: single tokens, odd sizes, tile edges, several tiles and a long inner sum
SHAPES = [(1, 1, 1), (1, 64, 128), (2, 8, 16), (3, 7, 5), (1, 1000, 3001), (16, 256, 512), (17, 520, 264), (48, 128, 1024), (64, 617, 1201),
          (127, 72, 96), (128, 128, 128), (129, 136, 200), (200, 1024, 384), (255, 520, 1000), (257, 264, 520), (300, 784, 300),
          (513, 96, 2056), (1003, 617, 1201), (2100, 256, 264), (40, 2048, 8192),
          (5000, 40, 72), (2, 1001, 2003), (7, 64, 4001), (8, 136, 40), (300, 64, 5000),
          # several tiles of tokens: all of them full, one token in the last, odd rows in all three matrices, and the sizes around a tile's
          (256, 768, 2048), (385, 512, 1024), (1500, 200, 1000), (130, 1537, 773), (4096, 72, 136), (4097, 136, 72),
          (33, 31, 65), (96, 64, 32), (9, 129, 33), (700, 33, 31)]
# an activation's FP32 value is off by a few steps: exp 2, its quotient 2, the products after it
ACT = 16 * E


def inputs(rows, cols, inner, t, pad=0, seed=0):
    x = rand((rows, cols), t, seed + 1, pad=pad)
    w = [rand((inner, cols), t, seed + 2, cols ** -0.5, pad=pad), rand((inner, cols), t, seed + 3, cols ** -0.5, pad=pad),
         rand((cols, inner), t, seed + 4, inner ** -0.5, pad=pad)]
    return x, w


def check_forward(got, x, w, act, t, h_round=1.0):
    x64, wg, wu, wd = x.double(), *(m.double() for m in w)
    gate, gate_err = product(x64, wg, 0, 0)
    up, up_err = product(x64, wu, 0, 0)
    a, da = act64(act, gate)
    h = a * up
    # |act''| <= 1.2 for all of them but relu, whose kink costs at most gate_err itself
    h_err = up.abs() * (da.abs() + 1) * gate_err + a.abs() * up_err + (ACT * (a.abs() + gate.abs() * ACT) * up.abs()) + E * h.abs()
    y, y_err = product(h, wd, h_err + h_round * u(t) * h.abs() + tiny(t), 0)
    within(got[0], y, y_err + u(t) * y.abs() + tiny(t), "y")
    if len(got) > 1:
        within(got[1], gate, gate_err + u(t) * gate.abs() + tiny(t), "gate")
        within(got[2], up, up_err + u(t) * up.abs() + tiny(t), "up")


def check_backward(got, dy, x, gate, up, w, act, t):
    dy, x, gate, up, wg, wu, wd = (m.double() for m in (dy, x, gate, up, *w))
    a, da = act64(act, gate)
    dh, dh_err = product(dy, wd.T, 0, 0)
    h, dgate, dup = a * up, dh * up * da, dh * a
    rel = u(t) + E
    slack = ACT * (a.abs() + gate.abs() * ACT)
    h_err = rel * h.abs() + tiny(t) + slack * up.abs()
    dgate_err = dh_err * (up * da).abs() + rel * dgate.abs() + tiny(t) + (dh * up).abs() * ACT * 2
    dup_err = dh_err * a.abs() + rel * dup.abs() + tiny(t) + slack * dh.abs()
    both = product(torch.cat([dgate, dup], 1), torch.cat([wg, wu], 0).T, torch.cat([dgate_err, dup_err], 1), 0)
    refs = [both, product(dgate.T, x.T, dgate_err.T, 0), product(dup.T, x.T, dup_err.T, 0), product(dy.T, h.T, 0, h_err.T)]
    for g, (ref, err), name in zip(got, refs, ("dx", "dw_gate", "dw_up", "dw_down")):
        within(g, ref, err + u(t) * ref.abs() + tiny(t), name)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("t", TYPES)
def test_forward(t, shape):
    t, act = TYPES[t], ACTS[sum(shape) % 5]
    x, w = inputs(*shape, t)
    got = gn.gated_ffn(x, *w, act=act, save=True)
    check_forward(got, x, w, act, t)
    alone = gn.gated_ffn(x, *w, act=act)
    check_forward((alone,), x, w, act, t)
    assert torch.equal(alone, gn.gated_ffn(x, *w, act=act))


@pytest.mark.parametrize("shape", [(1, 30, 37), (1, 1728, 25), (3, 64, 128), (17, 617, 1001), (128, 1024, 1024)])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_few_tokens_and_weights_keep_h(t, shape):
    """h in two parts: what is left of its rounding is half a step of a half step."""
    t = TYPES[t]
    for act in ACTS:
        x, w = inputs(*shape, t)
        check_forward(gn.gated_ffn(x, *w, act=act, save=True), x, w, act, t, h_round=u(t))


def test_h_beyond_the_type():
    """An h that FP16 cannot hold is infinite, with the sign that it has, and not NaN."""
    x, w = inputs(2, 16, 24, torch.float16)
    w[0].fill_(0); w[1].fill_(0); w[2].fill_(1)
    x[:, :2] = 256
    w[0][3, 0], w[1][3, 1] = 64, 64
    y, gate, up = gn.gated_ffn(x, *w, act="relu", save=True)
    assert bool((gate[:, 3] == 16384).all()) and bool((up[:, 3] == 16384).all())
    assert bool((y == float("inf")).all())
    w[1][3, 1] = -64
    assert bool((gn.gated_ffn(x, *w, act="relu") == -float("inf")).all())


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("t", TYPES)
def test_backward(t, shape):
    t, act = TYPES[t], ACTS[(sum(shape) + 1) % 5]
    x, w = inputs(*shape, t)
    dy = rand(shape[:2], t, 9, 0.5)
    _, gate, up = gn.gated_ffn(x, *w, act=act, save=True)
    got = gn.gated_ffn_grad(dy, x, gate, up, *w, act=act)
    check_backward(got, dy, x, gate, up, w, act, t)
    again = gn.gated_ffn_grad(dy, x, gate, up, *w, act=act)
    assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_more_rows_than_a_grid_has_tiles_in_its_second_dimension(t):
    """65535 tiles of 128 rows and one row."""
    t = TYPES[t]
    x, w = inputs(65535 * 128 + 1, 3, 5, t)
    dy = rand(x.shape, t, 9, 0.5)
    got = gn.gated_ffn(x, *w, save=True)
    check_forward(got, x, w, "silu", t)
    check_backward(gn.gated_ffn_grad(dy, x, got[1], got[2], *w), dy, x, got[1], got[2], w, "silu", t)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [5, 140])
@pytest.mark.parametrize("t", TYPES)
def test_activations(t, rows, act):
    t = TYPES[t]
    x, w = inputs(rows, 96, 160, t)
    w[0] *= 6                                       # gates from -20 to 20: both tails
    got = gn.gated_ffn(x, *w, act=act, save=True)
    check_forward(got, x, w, act, t)
    dy = rand((rows, 96), t, 9)
    check_backward(gn.gated_ffn_grad(dy, x, got[1], got[2], *w, act=act), dy, x, got[1], got[2], w, act, t)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [3, 200])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_gates_far_out_stay_finite(t, rows, act):
    """Gates of +-200: exp of them overflows FP32, the activations and their derivatives do not."""
    t = TYPES[t]
    x = torch.ones(rows, 8, dtype=t, device="cuda")
    w = [torch.full((16, 8), 25.0, dtype=t, device="cuda"), torch.ones(16, 8, dtype=t, device="cuda"), torch.ones(8, 16, dtype=t, device="cuda")]
    w[0][::2] = -25.0
    got = gn.gated_ffn(x, *w, act=act, save=True)
    check_forward(got, x, w, act, t)
    check_backward(gn.gated_ffn_grad(x, x, got[1], got[2], *w, act=act), x, x, got[1], got[2], w, act, t)


FAR = [60.0, 88.0, 100.0, 300.0, 1e3, 1e5, 1e9, 1e12, 1e15, 1e18, 1.8e19, 2e19, 1e20, 1e25, 1e30, 1e37]


def far_gates(rows, t, act, gates):
    """(y, dw_gate, dw_up) of gates of any size, with up = 1, weights and dy of ones: h = act(gate), dh = cols."""
    cols, inner = 8, len(gates)
    x = torch.zeros(rows, cols, dtype=t, device="cuda")
    x[:, 0] = 1
    one = lambda *shape: torch.ones(*shape, dtype=t, device="cuda")
    wg, wu = torch.zeros(inner, cols, dtype=t, device="cuda"), one(inner, cols)
    wg[:, 0] = torch.tensor(gates, dtype=torch.float64, device="cuda").to(t)
    y, gate, up = gn.gated_ffn(x, wg, wu, one(cols, inner), act=act, save=True)
    assert bool(((gate - wg[:, 0]).abs() <= 2.0 ** -18 * wg[:, 0].abs()).all()) and bool((up == 1).all())      # (FP32: two parts of 11 bits)
    dx, dwg, dwu, dwd = gn.gated_ffn_grad(one(rows, cols), x, gate, up, wg, wu, one(cols, inner), act=act)
    return y.double(), dwg[:, 0].double(), dwu[:, 0].double()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [3, 200, 5000])
def test_gates_far_below_leave_nothing(rows, act):
    """act and its derivative are zero, or below 1e-24, from -60 down to the type's last value.

    A sum of 16 such values, times cols = 8 and up to 5000 rows, and of their roundings: below 1e-18."""
    y, dwg, dwu = far_gates(rows, torch.bfloat16, act, [-v for v in FAR] + [-3e38])
    for m, name in ((y, "y"), (dwg, "dw_gate"), (dwu, "dw_up")):
        assert float(m.abs().max()) < 1e-18, (name, m.abs().max())


@pytest.mark.parametrize("act", ["sigmoid", "silu", "gelu"])
def test_tails_in_fp32(act):
    """One token, one column in use, the unit matrix behind it: y is the activation of each gate, and dw_gate its derivative.

    Relative to its terms each is off by the functions' own errors, at most 4 ulp of erfc and 2 of exp (8 E and 4 E), and five roundings; in
    both terms of a derivative."""
    n = 256
    v = torch.linspace(-12.5, 6.0, n, device="cuda")
    x = torch.zeros(1, n, device="cuda")
    x[0, 0] = 1
    wg, wu, wd = (torch.zeros(n, n, device="cuda") for _ in range(3))
    wg[:, 0], wu[:, 0] = v, 1
    wd.fill_diagonal_(1)
    y, gate, up = gn.gated_ffn(x, wg, wu, wd, act=act, save=True)
    assert torch.equal(gate[0], v) and bool((up == 1).all())
    dx, dwg, dwu, dwd = gn.gated_ffn_grad(torch.ones(1, n, device="cuda"), x, gate, up, wg, wu, wd, act=act)
    v = v.double()
    a, da = act64(act, v)
    if act == "gelu":                    # (Phi by erfc: torch's ndtr is 1 + erf in 64 bits too, and zero below -8.3)
        cdf, bell = 0.5 * torch.special.erfc(-v / math.sqrt(2)), v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        a, da, terms = v * cdf, cdf + bell, cdf + bell.abs()
    else:
        terms = (torch.special.expit(v) + v.abs() * torch.special.expit(v) * torch.special.expit(-v)) if act == "silu" else da
    within(y[0], a, 13 * E * a.abs() + tiny(torch.float32), "y")
    within(dwu[:, 0], a, 13 * E * a.abs() + tiny(torch.float32), "dw_up")
    within(dwg[:, 0], da, 13 * E * terms + tiny(torch.float32), "dw_gate")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [3, 200, 5000])
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_slopes_of_far_gates(t, rows, act):
    """The derivative is 1 far above (the sigmoid's 0), and 0 far below, to the rounding of a sum of `rows` equal terms cols = 8 and of dgate before it."""
    t = TYPES[t]
    for sign in (1, -1):
        _, dwg, _ = far_gates(rows, t, act, [sign * v for v in FAR])
        want = 8.0 * rows if sign > 0 and act != "sigmoid" else 0.0
        assert float((dwg - want).abs().max()) <= (2 * u(t) + rows * E) * want + 1e-18, (sign, dwg)


@pytest.mark.parametrize("pad", [1, 4, 8])
@pytest.mark.parametrize("rows", [2, 33, 300])
@pytest.mark.parametrize("t", TYPES)
def test_strides(t, rows, pad):
    t = TYPES[t]
    x, w = inputs(rows, 128, 192, t, pad)
    dy, gate, up = rand((rows, 128), t, 9, pad=pad), rand((rows, 192), t, 10, pad=pad), rand((rows, 192), t, 11, pad=pad)
    check_forward(gn.gated_ffn(x, *w, save=True), x, w, "silu", t)
    check_backward(gn.gated_ffn_grad(dy, x, gate, up, *w), dy, x, gate, up, w, "silu", t)


@pytest.mark.parametrize("offset", [1, 2, 4, 7])
@pytest.mark.parametrize("rows", [3, 150])
def test_misaligned_bases(rows, offset):
    t = torch.bfloat16
    cut = lambda r, c, seed, scale: rand((1, r * c + 8), t, seed, scale)[0][offset: offset + r * c].view(r, c)
    x, w = cut(rows, 64, 1, 1.0), [cut(136, 64, 2, 0.1), cut(136, 64, 3, 0.1), cut(64, 136, 4, 0.1)]
    y, gate, up = gn.gated_ffn(x, *w, save=True)
    check_forward((y, gate, up), x, w, "silu", t)
    check_backward(gn.gated_ffn_grad(x, x, gate, up, *w), x, x, gate, up, w, "silu", t)


def test_backward_against_differences():
    """Derivatives of sum(c * ffn) by central differences of the 64-bit form."""
    x, w = inputs(5, 6, 9, torch.float32)
    c = rand((5, 6), torch.float32, 7)
    for act in ("silu", "gelu", "gelu_tanh", "sigmoid"):
        _, gate, up = gn.gated_ffn(x, *w, act=act, save=True)
        got = gn.gated_ffn_grad(c, x, gate, up, *w, act=act)

        def f(x, wg, wu, wd):
            return float((((act64(act, x @ wg.T)[0] * (x @ wu.T)) @ wd.T) * c.double()).sum())

        at = [m.double() for m in (x, *w)]
        for which, g in enumerate(got):
            for k in range(0, g.numel(), 4):
                d = torch.zeros_like(at[which])
                d.view(-1)[k] = 1e-5
                up_, down = list(at), list(at)
                up_[which], down[which] = at[which] + d, at[which] - d
                # (error of the difference about 1e-10, of the call FP32 rounding of values up to about ten)
                assert abs((f(*up_) - f(*down)) / 2e-5 - float(g.view(-1)[k])) < 5e-5


@pytest.mark.parametrize("rows", [6, 300])
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_bad_rows_stay_to_themselves(t, rows):
    """A row with NaN or infinity spoils its own rows of y and dx and no other's.

    16-bit types: the others keep their bits.  FP32: what meets a cell of 128 x 128 elements with such an element is summed by FP32 FMAs
    instead of in two parts (gn_set_accurate_method), another order of the same terms: the others keep to the bounds of the 64-bit form."""
    t = TYPES[t]
    x, w = inputs(rows, 64, 128, t)
    y, gate, up = gn.gated_ffn(x, *w, save=True)
    dx = gn.gated_ffn_grad(x, x, gate, up, *w)[0]
    bad = x.clone()
    bad[2, 5], bad[4, 1] = float("nan"), float("inf")
    rest = [r for r in range(rows) if r not in (2, 4)]
    y2, gate2, up2 = gn.gated_ffn(bad, *w, save=True)
    assert bool(y2[2].isnan().all()) and not bool(y2[4].isfinite().any())
    dx2 = gn.gated_ffn_grad(bad, x, gate, up, *w)[0]
    assert bool(dx2[2].isnan().all())
    if t == torch.float32:
        check_forward((y2[rest], gate2[rest], up2[rest]), x[rest], w, "silu", t)
        check_backward((dx2[rest],), x[rest], x[rest], gate[rest], up[rest], w, "silu", t)
    else:
        assert torch.equal(y2[rest], y[rest]) and torch.equal(dx2[rest], dx[rest])


def test_no_rows():
    t = torch.bfloat16
    x, w = inputs(4, 24, 40, t)
    y, gate, up = gn.gated_ffn(x[:0], *w, save=True)
    assert y.shape == (0, 24) and gate.shape == (0, 40)
    dx, *dw = gn.gated_ffn_grad(x[:0], x[:0], gate, up, *w)
    assert dx.shape == (0, 24) and not any(bool(m.any()) for m in dw)


NAMES = ["x", "w_gate", "w_up", "w_down", "y", "gate", "up", "dy", "dx", "dw_gate", "dw_up", "dw_down"]


def raw(backward, kind, act, rows, cols, inner, mats):
    err = C.create_string_buffer(200)
    words = [v for n in NAMES for v in ((mats[n].data_ptr(), mats[n].stride(0)) if n in mats else (0, 0))]
    args = (C.c_int64 * 27)(kind | act << 32, rows, cols | inner << 32, *words)
    n = gn.lib().gn_gated_ffn_workspace(args, backward)
    assert n > 0
    ws = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    fn = gn.lib().gn_gated_ffn_grad if backward else gn.lib().gn_gated_ffn
    assert fn(args, ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream, err, 200) == 0, err.value
    assert bool((ws[n:] == 0x5A).all())             # nothing behind the workspace


@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("rows,cols,inner", [(3, 100, 72), (130, 65, 129), (300, 256, 136)])
@pytest.mark.parametrize("t", TYPES)
def test_what_is_left_alone_and_outputs_not_wanted(t, rows, cols, inner, pad):
    """Outputs in wider buffers: what lies past a row's end and behind the last row stays; an output that is not wanted is left out."""
    kind, t = {"f32": 0, "bf16": 1, "f16": 2}[t], TYPES[t]
    x, w = inputs(rows, cols, inner, t)
    dy = rand((rows, cols), t, 9)
    y, gate, up = gn.gated_ffn(x, *w, act="gelu", save=True)
    want = dict(zip(NAMES[8:], gn.gated_ffn_grad(dy, x, gate, up, *w, act="gelu")), y=y, gate=gate, up=up)
    shapes = dict(y=(rows, cols), gate=(rows, inner), up=(rows, inner), dx=(rows, cols), dw_gate=(inner, cols), dw_up=(inner, cols), dw_down=(cols, inner))
    ins = dict(x=x, w_gate=w[0], w_up=w[1], w_down=w[2])

    def outputs(names):
        return {n: torch.full((shapes[n][0] + 2, shapes[n][1] + pad), 7.0, dtype=t, device="cuda") for n in names}

    def compare(out):
        for n, b in out.items():
            r, c = shapes[n]
            assert torch.equal(b[:r, :c], want[n]), n
            assert bool((b[r:] == 7).all()) and bool((b[:, c:] == 7).all()), n

    for names in (["y"], ["y", "gate"], ["y", "up"], ["y", "gate", "up"]):
        out = outputs(names)
        raw(0, kind, 2, rows, cols, inner, dict(ins, **out))
        compare(out)
    for names in (["dx"], ["dw_gate"], ["dw_up", "dw_down"], ["dx", "dw_gate", "dw_up", "dw_down"], []):
        out = outputs(names)
        raw(1, kind, 2, rows, cols, inner, dict(ins, gate=gate, up=up, dy=dy, **out))
        compare(out)


@pytest.mark.parametrize("pad", [0, 1, 3])
@pytest.mark.parametrize("rows,cols,inner", [(4200, 130, 203), (700, 1001, 1300)])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_large_tiles_of_unaligned_rows(t, rows, cols, inner, pad):
    """Rows of outputs that start at every even byte of 16, in whole and in cut chunks of columns, and what lies around them."""
    kind, t = {"bf16": 1, "f16": 2}[t], TYPES[t]
    x, w = inputs(rows, cols, inner, t)
    dy = rand((rows, cols), t, 9)
    shapes = dict(y=(rows, cols), gate=(rows, inner), up=(rows, inner), dx=(rows, cols), dw_gate=(inner, cols), dw_up=(inner, cols), dw_down=(cols, inner))
    ins = dict(x=x, w_gate=w[0], w_up=w[1], w_down=w[2])
    whole = {n: torch.full(((s[0] + 2) * (s[1] + pad) + 1,), 7.0, dtype=t, device="cuda") for n, s in shapes.items()}
    out = {n: b[1:].view(shapes[n][0] + 2, shapes[n][1] + pad) for n, b in whole.items()}        # (bases off by one element)
    got = {n: b[:shapes[n][0], :shapes[n][1]] for n, b in out.items()}
    raw(0, kind, 2, rows, cols, inner, dict(ins, **{n: out[n] for n in ("y", "gate", "up")}))
    check_forward([got[n] for n in ("y", "gate", "up")], x, w, "gelu", t)
    raw(1, kind, 2, rows, cols, inner, dict(ins, dy=dy, **{n: out[n] for n in shapes if n != "y"}))
    check_backward([got[n] for n in ("dx", "dw_gate", "dw_up", "dw_down")], dy, x, got["gate"], got["up"], w, "gelu", t)
    for n, (r, c) in shapes.items():
        assert whole[n][0] == 7 and bool((out[n][r:] == 7).all()) and bool((out[n][:, c:] == 7).all()), n


def test_refusals():
    x, w = inputs(4, 16, 24, torch.bfloat16)
    _, gate, up = gn.gated_ffn(x, *w, save=True)
    for bad in (lambda: gn.gated_ffn(x.double(), *w), lambda: gn.gated_ffn(x, w[0].half(), w[1], w[2]), lambda: gn.gated_ffn(x, w[0], w[1].cpu(), w[2]),
                lambda: gn.gated_ffn_grad(x.float(), x, gate, up, *w), lambda: gn.gated_ffn_grad(x, x, gate.float(), up, *w)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: gn.gated_ffn(x, *w, act="tanh"), lambda: gn.gated_ffn(x, w[0], w[1], w[0]), lambda: gn.gated_ffn(x, w[0][:20], w[1], w[2]),
                lambda: gn.gated_ffn(x[0], *w), lambda: gn.gated_ffn(x, w[0].T, w[1], w[2]), lambda: gn.gated_ffn(x, w[0][:0], w[1][:0], w[2][:, :0]),
                lambda: gn.gated_ffn_grad(x[:3], x, gate, up, *w), lambda: gn.gated_ffn_grad(x, x, gate[:, :8], up, *w)):
        with pytest.raises(ValueError):
            bad()


def test_saved_rows_start_on_16_bytes():
    for t in (torch.bfloat16, torch.float32):
        x, w = inputs(5, 16, 27, t)
        _, gate, up = gn.gated_ffn(x, *w, save=True)
        for m in (gate, up):
            assert m.shape == (5, 27) and m.stride(1) == 1 and m.stride(0) == (27 if t is torch.float32 else 32)


def test_status_after_calls():
    x, w = inputs(300, 64, 128, torch.bfloat16)
    gn.gated_ffn(x, *w)
    gn.gated_ffn_status()
    gn.gated_ffn_status(stream=torch.cuda.Stream())


@pytest.mark.parametrize("rows", [1, 100, 700])
def test_same_tensor_in_several_places(rows):
    """One matrix as gate and up projection, and one as x and dy."""
    for t in (torch.bfloat16, torch.float32):
        x, w = inputs(rows, 128, 256, t)
        w[1] = w[0]
        got = gn.gated_ffn(x, *w, save=True)
        check_forward(got, x, w, "silu", t)
        check_backward(gn.gated_ffn_grad(x, x, got[1], got[1], *w), x, x, got[1], got[1], w, "silu", t)

