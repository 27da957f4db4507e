"""Layer norm and its backward pass against a plain form in 64 bits."""
import ctypes as C
import math

import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import E, TYPES, rand, tiny, u, vec, within

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (5, 2), (3, 7), (131, 8), (33, 33), (257, 64), (1, 100), (700, 127), (64, 256), (300, 617), (19, 1000), (4001, 1024),
          (7, 1201), (40, 4096), (3, 8200), (2, 16384), (2, 16385), (3, 32768), (2, 70001), (1, 300000)]


def norm64(x, w, b, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = (d.square().mean(1, keepdim=True) + eps) ** -0.5
    y = d * rstd * (1 if w is None else w.double()) + (0 if b is None else b.double())
    return y, mean[:, 0], rstd[:, 0]


def norm_bounds(x, w, b, y, mean, rstd, t):
    """FP32 arithmetic on a row: sums of up to cols / 32 terms a thread in sequence and a tree of 10 steps after it (each term of the sums
    carries one or two roundings), rstd of a quotient, a root and a reciprocal, and the four operations of y."""
    n = x.shape[1]
    rel = E * (n / 32 + 24)
    x = x.double()
    spread = x.abs().mean(1)                                       # what the sum's roundings are relative to
    m_err = rel * (x - mean[:, None]).abs().mean(1) + 2 * E * mean.abs() + (E * (n / 32 + 24)) ** 2 * spread
    r_err = rel * rstd
    W = torch.ones_like(x) if w is None else w.double().expand_as(x)
    B = torch.zeros_like(x) if b is None else b.double().expand_as(x)
    scaled = (x - mean[:, None]).abs() * rstd[:, None] * W.abs()
    y_err = u(t) * y.abs() + tiny(t) + (rel + 4 * E) * scaled + 2 * E * B.abs() + (m_err - 2 * E * mean.abs())[:, None] * rstd[:, None] * W.abs() \
        + E * (x.abs() + mean.abs()[:, None]) * rstd[:, None] * W.abs() * (E * n)
    return y_err, m_err + 1e-30, r_err


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("t,wt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
def test_forward(t, wt, shape):
    rows, cols = shape
    t, wt = TYPES[t], TYPES[wt]
    x = rand(shape, t, rows + cols, 1.5, 0.3)
    w, b = vec(cols, wt, 1, 0.2, 1.0), vec(cols, wt, 2, 0.3)
    y, mean, rstd = gn.layer_norm(x, w, b, 1e-5, save=True)
    ry, rm, rr = norm64(x, w, b, 1e-5)
    by, bm, br = norm_bounds(x, w, b, ry, rm, rr, t)
    within(y, ry, by, "y")
    within(mean, rm, bm, "mean")
    within(rstd, rr, br, "rstd")
    assert torch.equal(gn.layer_norm(x, w, b, 1e-5), y)


@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("w,b", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("t", TYPES)
def test_forward_strides_and_no_weights(t, w, b, pad):
    t = TYPES[t]
    x = rand((57, 520), t, 3, 1.0, -0.5, pad)
    w, b = vec(520, t, 1) if w else None, vec(520, t, 2) if b else None
    y, mean, rstd = gn.layer_norm(x, w, b, 0.0, save=True)
    ry, rm, rr = norm64(x, w, b, 0.0)
    by, _, _ = norm_bounds(x, w, b, ry, rm, rr, t)
    within(y, ry, by, "y")


@pytest.mark.parametrize("offset", range(1, 8))
def test_forward_misaligned_bases(offset):
    flat = vec(64 * 1024 + 8, torch.bfloat16, 4)
    w = vec(1024 + 8, torch.bfloat16, 5)
    x = flat[offset: offset + 64 * 1024].view(64, 1024)
    b = w[8 - offset: 8 - offset + 1024]
    w = w[offset: offset + 1024]
    y, mean, rstd = gn.layer_norm(x, w, b, save=True)
    ry, rm, rr = norm64(x, w, b, 1e-5)
    by, bm, br = norm_bounds(x, w, b, ry, rm, rr, torch.bfloat16)          # (rows that 16-byte loads cannot read are summed in another order)
    within(y, ry, by, "y")
    within(mean, rm, bm, "mean")
    within(rstd, rr, br, "rstd")


def test_forward_of_a_large_mean():
    """mean / spread = 10^4: the corrected sums keep y to FP32 accuracy of the values x - mean, which are exact to 2^-24 |x|."""
    x = rand((40, 3000), torch.float32, 6, 1.0, 1e4)
    y, mean, rstd = gn.layer_norm(x, save=True)
    ry, rm, rr = norm64(x, None, None, 1e-5)
    # x - m is exact (Sterbenz) and the correction removes m's own error; what is left is rel of the spread
    within(y, ry, E * (3000 / 32 + 40) * (ry.abs() + 1), "y")
    within(mean, rm, 2 * E * rm.abs(), "mean")
    within(rstd, rr, E * (3000 / 32 + 40) * rr, "rstd")


@pytest.mark.parametrize("cols", [5, 640, 4096, 20000])
def test_forward_rows_of_equal_elements_and_bad_rows(cols):
    x = rand((6, cols), torch.float32, 7)
    good = gn.layer_norm(x)
    x[1] = 3.25
    x[3, cols // 2] = float("nan")
    x[4, cols - 1] = float("inf")
    y, mean, rstd = gn.layer_norm(x, save=True)
    assert torch.equal(y[[0, 2, 5]], good[[0, 2, 5]])
    assert bool((y[1] == 0).all()) and float(mean[1]) == 3.25 and abs(float(rstd[1]) - 1e-5 ** -0.5) < 1e-3
    assert bool(y[3].isnan().all()) and bool(y[4].isnan().any())


@pytest.mark.parametrize("eps", [1e-5, 1e-12])
@pytest.mark.parametrize("cols", [5, 33, 100, 500, 617, 1001, 1201, 4097, 9001, 20001, 300000, 1 << 20])
def test_forward_of_equal_elements_whose_sum_is_not_exact(cols, eps):
    """A row of n times v has the mean v, no variance and the bias, whatever the sum of n v is rounded to.

    The sums are taken about the row's first element, so they are zero: y is b and the mean v.  rstd: eps in FP32, the root, the quotient."""
    values = [v * s for v in (1e3, 1.7e4, 1e5, 1e6, 1.9e7, 122624096.0, 1.2345e9, 2.9e9, 1e25, 0.1) for s in (1, -1.0001)] + [3e38]
    x = torch.tensor(values, dtype=torch.float64, device="cuda").float()[:, None].repeat(1, cols)
    w, b = vec(cols, torch.float32, 1, 0.2, 1.0), vec(cols, torch.float32, 2, 0.3)
    y, mean, rstd = gn.layer_norm(x, w, b, eps, save=True)
    within(rstd, torch.full((len(values),), eps ** -0.5, dtype=torch.float64, device="cuda"), 4 * E * torch.full((1,), eps ** -0.5, device="cuda"), "rstd")
    assert torch.equal(mean, x[:, 0]) and bool((y == b).all())


@pytest.mark.parametrize("eps", [1e-5, 1e-12])
@pytest.mark.parametrize("cols", [5, 33, 100, 500, 617, 1001, 1201, 4097, 8191, 9001, 20001, 40001])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_forward_of_equal_elements_in_16_bits(t, cols, eps):
    """The same, over every mantissa of BF16 and an eighth of FP16's, at two ends of the exponents."""
    t = TYPES[t]
    top = torch.arange(1024, 2048, 8, device="cuda").double() / 2048
    x = torch.cat([top * (65504.0 if t == torch.float16 else 2.0 ** 40), top * -0.125]).to(t)[:, None].repeat(1, cols)
    b = vec(cols, torch.float32, 2, 0.3)
    y, mean, rstd = gn.layer_norm(x, None, b, eps, save=True)
    within(rstd, torch.full((256,), eps ** -0.5, dtype=torch.float64, device="cuda"), 4 * E * torch.full((1,), eps ** -0.5, device="cuda"), "rstd")
    assert torch.equal(mean, x[:, 0].float()) and bool((y == b.to(t)).all())


@pytest.mark.parametrize("cols", [7, 64, 250, 1001, 3001, 9001, 20001])
@pytest.mark.parametrize("v", [1e4, 1e6, 1.2345e9])
def test_forward_of_a_spread_of_a_few_steps(cols, v):
    """Elements within three steps of FP32 of one another beside rows of equal ones: x - m and its sums are exact, (sum)^2 / n but for E^2 of it, so the
    bounds are those of the values x - mean."""
    x = torch.full((12, cols), v, dtype=torch.float32, device="cuda")
    step = 2.0 ** (math.floor(math.log2(v)) - 23)
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    x[::2] += torch.randint(-1, 3, (6, cols), generator=g, device="cuda") * step
    x[4], x[4, cols // 2] = v, v + step
    eps = (step * 1e-3) ** 2
    y, mean, rstd = gn.layer_norm(x, eps=eps, save=True)
    ry, rm, rr = norm64(x, None, None, eps)
    rel = E * (cols / 32 + 40)
    within(rstd, rr, rel * rr, "rstd")
    within(mean, rm, 2 * E * rm.abs(), "mean")
    within(y, ry, rel * (ry.abs() + 1), "y")


def grads64(dy, x, mean, rstd, w, add):
    dy, xh = dy.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy if w is None else dy * w.double()
    dx = rstd.double()[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx + (0 if add is None else add.double()), (dy * xh).sum(0), dy.sum(0)


def check_grads(got, dy, x, mean, rstd, w, add, t, wt):
    n, rows = x.shape[1], x.shape[0]
    ref = grads64(dy, x, mean, rstd, w, add)
    xh = ((x.double() - mean.double()[:, None]) * rstd.double()[:, None]).abs()
    g = dy.double().abs() * (1 if w is None else w.double().abs())
    rel, rs = E * (n / 32 + 24), rstd.double()[:, None]
    x_err = E * (x.double().abs() + mean.double().abs()[:, None]) * rs          # of (x - mean) rstd, absolute
    # every term of dx with the roundings that went into it, the sums with theirs
    b_dx = u(t) * ref[0].abs() + tiny(t) + 6 * E * rs * g + rs * rel * (g.mean(1, keepdim=True) + xh * (g * xh).mean(1, keepdim=True)) \
        + rs * (x_err * (g * xh).mean(1, keepdim=True) + xh * (g * x_err).mean(1, keepdim=True)) + 2 * E * (0 if add is None else add.double().abs())
    within(got[0], ref[0], b_dx, "dx")
    if len(got) == 1:
        return
    # sums over rows: every addition is off by at most E of a partial sum, in sequence over the rows of a block and then over the blocks
    terms = dy.double().abs() * xh
    acc = 7 * E * max(rows, 1) ** 0.5 + 8 * E
    spread = lambda v: (v * v).sum(0).sqrt()
    b_dw = u(wt) * ref[1].abs() + tiny(wt) + acc * (ref[1].abs() + 7 * spread(terms)) + (dy.double().abs() * x_err).sum(0) + 4 * E * terms.sum(0)
    within(got[1], ref[1], b_dw, "dweight")
    b_db = u(wt) * ref[2].abs() + tiny(wt) + acc * (ref[2].abs() + 7 * spread(dy.double()))
    within(got[2], ref[2], b_db, "dbias")


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("shape", SHAPES + [(20000, 96), (9000, 24), (5000, 520)])
@pytest.mark.parametrize("t,wt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
def test_backward(t, wt, shape, add):
    rows, cols = shape
    t, wt = TYPES[t], TYPES[wt]
    x = rand(shape, t, rows + 3 * cols, 1.5, 0.3)
    dy = rand(shape, t, rows + 5 * cols, 0.5)
    w = vec(cols, wt, 1, 0.2, 1.0)
    a = rand(shape, t, 9) if add else None
    _, mean, rstd = gn.layer_norm(x, w, save=True)
    got = gn.layer_norm_grad(dy, x, mean, rstd, w, add=a)
    assert got[0].dtype == t and got[1].dtype == wt and got[2].dtype == wt
    check_grads(got, dy, x, mean, rstd, w, a, t, wt)
    again = gn.layer_norm_grad(dy, x, mean, rstd, w, add=a)
    assert all(torch.equal(p, q) for p, q in zip(got, again))          # sums in a fixed order


@pytest.mark.parametrize("cols", [24, 521, 5000])
@pytest.mark.parametrize("t", TYPES)
def test_backward_strides_and_no_weight(t, cols):
    t = TYPES[t]
    x, dy, add = rand((77, cols), t, 1, pad=3), rand((77, cols), t, 2, pad=1), rand((77, cols), t, 3, pad=8)
    _, mean, rstd = gn.layer_norm(x, save=True)
    check_grads(gn.layer_norm_grad(dy, x, mean, rstd, None, add=add), dy, x, mean, rstd, None, add, t, t)


def test_backward_against_differences():
    """d/dx of sum(c * norm(x)) by central differences of the 64-bit form."""
    x, w, c = rand((3, 17), torch.float32, 1), vec(17, torch.float32, 2, 0.2, 1.0), rand((3, 17), torch.float32, 3)
    _, mean, rstd = gn.layer_norm(x, w, save=True)
    dx, dw, db = gn.layer_norm_grad(c, x, mean, rstd, w)
    h, x64 = 1e-5, x.double()
    f = lambda x, w: (norm64(x, w, None, 1e-5)[0] * c.double()).sum()
    for i in range(3):
        for j in range(17):
            d = torch.zeros_like(x64)
            d[i, j] = h
            # the difference's own error is of the order h^2 = 1e-10 and 1e-16 / h = 1e-11; the call's is FP32 rounding
            assert abs(float((f(x64 + d, w) - f(x64 - d, w)) / (2 * h)) - float(dx[i, j])) < 2e-5
    for j in range(17):
        d = torch.zeros(17, dtype=torch.float64, device="cuda")
        d[j] = h
        assert abs(float((f(x64, w.double() + d) - f(x64, w.double() - d)) / (2 * h)) - float(dw[j])) < 2e-5


def test_no_rows():
    x = torch.empty(0, 40, dtype=torch.bfloat16, device="cuda")
    w = vec(40, torch.float32, 1)
    y, mean, rstd = gn.layer_norm(x, w, save=True)
    assert y.shape == (0, 40) and mean.shape == (0,)
    dx, dw, db = gn.layer_norm_grad(x, x, mean, rstd, w)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()


@pytest.mark.parametrize("pad", [5, 8])
@pytest.mark.parametrize("cols", [12, 24, 600, 4096, 9000, 40000])
def test_in_place_and_what_is_left_alone(cols, pad):
    """y in x's place, dx in dy's and in add's; columns past the row's end and rows behind the last keep what they hold.  More rows than a
    launch has blocks, so that blocks walk several."""
    rows, ld = 9 if cols > 600 else 1500, cols + pad
    err = C.create_string_buffer(200)
    x, dy, add = rand((rows, cols), torch.float16, 1), rand((rows, cols), torch.float16, 2), rand((rows, cols), torch.float16, 3)
    w = vec(cols, torch.float16, 4)
    def wide(m):
        b = torch.full((rows + 2, ld), 7.0, dtype=torch.float16, device="cuda")
        b[:rows, :cols] = m
        return b

    def kept(b):
        assert bool((b[rows:] == 7).all()) and bool((b[:, cols:] == 7).all())
        return b[:rows, :cols]

    bx, by = wide(x), wide(torch.zeros_like(x))
    _, mean, rstd = gn.layer_norm(bx[:rows, :cols], w, save=True)
    for out in (by, bx):
        assert gn.lib().gn_layer_norm(2, 2, rows, cols, bx.data_ptr(), ld, w.data_ptr(), None, 1e-5, out.data_ptr(), ld, None, None,
                                      torch.cuda.current_stream().cuda_stream, err, 200) == 0, err.value
    assert torch.equal(kept(bx), kept(by)) and bool(by[:rows, :cols].any())
    n = gn.lib().gn_layer_norm_grad_workspace(rows, cols)
    ws = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    got, bx = [], wide(x)
    for place in (2, 0, 1):
        b = [wide(dy), wide(add), wide(torch.zeros_like(dy))]
        assert gn.lib().gn_layer_norm_grad(2, 2, rows, cols, b[0].data_ptr(), ld, bx.data_ptr(), ld, mean.data_ptr(), rstd.data_ptr(), w.data_ptr(),
                                           b[1].data_ptr(), ld, b[place].data_ptr(), ld, None, None, ws.data_ptr(), n,
                                           torch.cuda.current_stream().cuda_stream, err, 200) == 0, err.value
        got.append(kept(b[place]))
        assert all(bool((kept(b[k]) == (dy, add)[k]).all()) for k in range(2) if k != place)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    check_grads((got[0],), dy, x, mean, rstd, w, add, torch.float16, torch.float16)
    assert bool((ws[n:] == 0x5A).all())


def test_refusals():
    x = rand((4, 16), torch.bfloat16, 1)
    _, mean, rstd = gn.layer_norm(x, save=True)
    for bad in (lambda: gn.layer_norm(x.double()), lambda: gn.layer_norm(x, vec(16, torch.float16, 1)),
                lambda: gn.layer_norm(x, vec(16, torch.float32, 1), vec(16, torch.bfloat16, 1)),
                lambda: gn.layer_norm_grad(x.float(), x, mean, rstd), lambda: gn.layer_norm_grad(x, x, mean.double(), rstd),
                lambda: gn.layer_norm_grad(x, x, None, rstd)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: gn.layer_norm(x[0]), lambda: gn.layer_norm(x, vec(15, torch.bfloat16, 1)), lambda: gn.layer_norm(x.T),
                lambda: gn.layer_norm(x[:1].expand(4, 16)), lambda: gn.layer_norm(x[:, :0]), lambda: gn.layer_norm_grad(x[:3], x, mean, rstd),
                lambda: gn.layer_norm_grad(x, x, mean[:3], rstd), lambda: gn.layer_norm_grad(x, x, mean, rstd, add=x[:, :8])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(gn.GnError, match="eps"):
        gn.layer_norm(x, eps=-1.0)


def test_rows_too_long_are_refused_by_the_library():
    x = torch.zeros(1, (1 << 20) + 1, dtype=torch.bfloat16, device="cuda")
    one = torch.ones(1, device="cuda")
    for call in (lambda: gn.layer_norm(x), lambda: gn.layer_norm_grad(x, x, one, one)):
        with pytest.raises(gn.GnError, match="cols must be in"):
            call()
