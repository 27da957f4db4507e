"""A mixture of experts in the place of a block's feed-forward layer, as a training step and a decoder use it:
out = x + sum over the chosen experts of weight * ffn_expert(norm(x)), the choice by route on the norm's logits."""
import threading

import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import TYPES, act64, rand, vec
from mixture_common import used, weights_of

pytestmark = pytest.mark.gpu

ROUTER = dict(score="sigmoid", renormalise=True, scale=1.5)


def parameters(cols, inner, experts, t):
    w = weights_of(experts, cols, inner, t)
    return dict(w=vec(cols, t, 1, 0.1, 1.0), b=vec(cols, t, 2, 0.1), router=rand((experts, cols), t, 3, cols ** -0.5), bias=vec(experts, torch.float32, 4, 0.05),
                gate=w[0], up=w[1], down=w[2])


def library(a, b):
    return a @ b.T


def by_hand(a, b):
    return (a.float()[:, None] * b.float()).sum(-1).to(a.dtype)


def choose(h, q, k, stream=None, product=library):
    """(logits, index, weight); the router's product is the user's own, in the type."""
    with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
        logits = product(h, q["router"])
    index, weight = gn.route(logits, k, bias=q["bias"], groups=2, top_groups=1, group_best=2, stream=stream, **ROUTER)
    return logits, index, weight


def forward(x, q, k, stream=None, product=library):
    h, mean, rstd = gn.layer_norm(x, q["w"], q["b"], save=True, stream=stream)
    logits, index, weight = choose(h, q, k, stream, product)
    y, gate, up = gn.experts(h, index, weight, q["gate"], q["up"], q["down"], save=True, stream=stream)
    return gn.dropout(y, 0.0, 1, residual=x, stream=stream), (h, mean, rstd, logits, index, weight, gate, up)


def backward(dout, x, q, kept, stream=None, product=library):
    h, mean, rstd, logits, index, weight, gate, up = kept
    dh, dweight, *dw = gn.experts_grad(dout, h, index, weight, gate, up, q["gate"], q["up"], q["down"], stream=stream)
    dlogits = gn.route_grad(dweight, logits, index, stream=stream, **ROUTER)
    with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
        dh2, drouter = dh + product(dlogits, q["router"].T), product(dlogits.T, h.T)
    dx, dnw, dnb = gn.layer_norm_grad(dh2, x, mean, rstd, q["w"], add=dout, stream=stream)
    return [dx, dnw, dnb, drouter, *dw]


def block64(x, q, index):
    d = x - x.mean(1, keepdim=True)
    h = d * (d.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * q["w"] + q["b"]
    s = torch.sigmoid(h @ q["router"].T).gather(1, index.long())
    s = s / s.sum(1, keepdim=True) * 1.5
    y = x.clone()
    for e, t, j in used(index, q["gate"].shape[0]):
        y = y.index_put((t,), s[t, j][:, None] * ((act64("silu", h[t] @ q["gate"][e].T)[0] * (h[t] @ q["up"][e].T)) @ q["down"][e].T), accumulate=True)
    return y


NAMES = ("w", "b", "router", "gate", "up", "down")


@pytest.mark.parametrize("rows,cols,inner,experts,k", [(1, 64, 96, 4, 2), (40, 136, 77, 8, 3), (300, 256, 520, 4, 1), (1000, 520, 264, 16, 4)])
@pytest.mark.parametrize("t", TYPES)
def test_block_and_its_gradients(t, rows, cols, inner, experts, k):
    """Against automatic differentiation of the 64-bit form, on the choice that the block has made.

    Each value has at most seven roundings to the type behind it (norm, logits, projection or h, y, and dh, dlogits, dgate and their sum in the backward pass), independent
    and of at most u each: in the 2-norm they stay below 7 u of the result times the gain of what follows, about one here."""
    t = TYPES[t]
    q, x, dout = parameters(cols, inner, experts, t), rand((rows, cols), t, 6), rand((rows, cols), t, 7)
    out, kept = forward(x, q, k)
    got = backward(dout, x, q, kept)
    leaves = [x.double().requires_grad_()] + [q[n].double().requires_grad_() for n in NAMES]
    ref = block64(leaves[0], dict(zip(NAMES, leaves[1:])), kept[4])
    grads = torch.autograd.grad(ref, leaves, dout.double())
    limit = 7 * torch.finfo(t).eps / 2 if t != torch.float32 else 3e-6
    for g, r, name in zip([out] + got, (ref.detach(), *grads), ("out", "dx", "dnorm_w", "dnorm_b", "drouter", "dw_gate", "dw_up", "dw_down")):
        if name == "drouter" and k == 1:                     # (one weight, divided by itself: a gradient of nothing but roundings)
            continue
        off = float((g.double() - r).norm() / r.norm())
        assert off < limit, (name, off)


def test_other_streams_and_two_at_once():
    """The block on two streams at the same time, from two threads, gives what it gives alone."""
    t = torch.bfloat16
    q = parameters(256, 136, 8, t)
    xs, douts = [rand((400, 256), t, s) for s in (1, 2)], [rand((400, 256), t, s) for s in (3, 4)]
    want = []
    for x, d in zip(xs, douts):
        out, kept = forward(x, q, 2)
        want.append([out] + backward(d, x, q, kept))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]

    def work(n):
        for _ in range(20):
            out, kept = forward(xs[n], q, 2, stream=streams[n])
            got[n] = [out] + backward(douts[n], xs[n], q, kept, stream=streams[n])

    threads = [threading.Thread(target=work, args=(n,)) for n in range(2)]
    [th.start() for th in threads]
    [th.join() for th in threads]
    torch.cuda.synchronize()
    for n in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[n], want[n]))
    gn.gated_ffn_status()


@pytest.mark.parametrize("t", TYPES)
def test_captured_training_step(t):
    """Two graphs of the same step, replayed at once on changing inputs, against eager calls.  The router's products are sums of torch's here: products of its library in
    two graphs share one workspace, in which the kernels count and wait for their slices of K, so graphs that hold them must not run at once."""
    t = TYPES[t]
    q = parameters(264, 72, 6, t)
    xs, dout = [rand((300, 264), t, s) for s in (1, 2)], rand((300, 264), t, 3)

    def step(x):
        out, kept = forward(x, q, 2, product=by_hand)
        return [out] + backward(dout, x, q, kept, product=by_hand)

    step(xs[0])
    graphs, outs = [], []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(x))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for n in range(3):
        for s, x in enumerate(xs):
            x.copy_(rand(x.shape, t, 10 * n + s))
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for x, got in zip(xs, outs):
            assert all(torch.equal(a, b) for a, b in zip(got, step(x)))
    gn.gated_ffn_status()


def test_padded_batch():
    """Tokens that are padding go to no expert: theirs is the residual, and nothing of theirs is in a gradient."""
    t = torch.bfloat16
    q, x, dout = parameters(136, 72, 8, t), rand((50, 136), t, 6), rand((50, 136), t, 7)
    h = gn.layer_norm(x, q["w"], q["b"])
    _, index, weight = choose(h, q, 2)
    _, short, _ = choose(h[:30], q, 2)
    index[30:] = -1
    assert torch.equal(index[:30], short)
    y, gate, up = gn.experts(h, index, weight, q["gate"], q["up"], q["down"], save=True)
    dh, dweight, *dw = gn.experts_grad(dout, h, index, weight, gate, up, q["gate"], q["up"], q["down"])
    y2, gate2, up2 = gn.experts(h[:30], short, weight[:30], q["gate"], q["up"], q["down"], save=True)
    dh2, dweight2, *dw2 = gn.experts_grad(dout[:30], h[:30], short, weight[:30], gate2, up2, q["gate"], q["up"], q["down"])
    assert bool((y[30:] == 0).all()) and bool((dh[30:] == 0).all()) and bool((dweight[30:] == 0).all())
    assert torch.equal(y[:30], y2) and torch.equal(dh[:30], dh2) and torch.equal(dweight[:30], dweight2) and all(torch.equal(a, b) for a, b in zip(dw, dw2))


@pytest.mark.parametrize("t", TYPES)
def test_decoder_on_4_bit_weights(t):
    """The experts of a batch of decoders on 4-bit weights, and on what these stand for in the type: h rounded to 17 bits or more in one form and to the type in the
    other, both to the type at the end, so three half steps at most, independent, and the type's rounding of the weights, a half step of each."""
    t = TYPES[t]
    q, x = parameters(256, 136, 8, t), rand((9, 256), t, 6)
    h = gn.layer_norm(x, q["w"], q["b"])
    _, index, weight = choose(h, q, 3)
    w = [gn.quantize4(q[n], 32) for n in ("gate", "up", "down")]
    got = gn.gated_ffn4(h, *w, index=index, weight=weight)
    want = gn.experts(h, index, weight, *(gn.unpack4(m) for m in w))
    limit = 4 * torch.finfo(t).eps / 2 if t != torch.float32 else 2e-6
    assert float((got.double() - want.double()).norm() / want.double().norm()) < limit


def test_arguments_dropped_after_a_call_on_another_stream():
    """Their memory is not handed out again before that stream has read it: the calls wait behind a pause of some 50 ms, while the current
    stream allocates tensors of the same sizes and fills them."""
    t = torch.bfloat16
    q, side, x, dout = parameters(256, 136, 8, t), torch.cuda.Stream(), rand((60, 256), t, 1), rand((60, 256), t, 2)
    logits, index, weight = choose(x, q, 2)
    _, gate, up = gn.experts(x, index, weight, q["gate"], q["up"], q["down"], save=True)
    dweight, W = rand((60, 2), torch.float32, 5), (q["gate"], q["up"], q["down"])
    W4 = [gn.quantize4(m, 32) for m in W]
    calls = [(lambda a, s: gn.route(a[0], 2, bias=a[1], stream=s), (logits, q["bias"])), (lambda a, s: gn.route_grad(*a, stream=s), (dweight, logits, index)),
             (lambda a, s: gn.experts(*a, stream=s), (x, index, weight, *W)), (lambda a, s: gn.experts_grad(*a, stream=s), (dout, x, index, weight, gate, up, *W)),
             (lambda a, s: gn.gated_ffn4(a[0], *a[3:], index=a[1], weight=a[2], stream=s), (x, index, weight, *W4))]
    copy = lambda a: gn.Weight4(a.q.clone(), a.scale.clone(), a.experts, a.rows, a.cols, a.group) if isinstance(a, gn.Weight4) else a.clone()
    flat = lambda a: [m for n in a for m in ((n.q, n.scale) if isinstance(n, gn.Weight4) else (n,))]
    for call, args in calls:
        want = call(args, None)
        mine = [copy(a) for a in args]
        places = {a.data_ptr(): (a.shape, a.dtype) for a in flat(mine)}
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        got = call(mine, side)
        del mine
        over = []
        for shape, dtype in [v for v in places.values() for _ in range(4)]:
            over.append(torch.full(shape, 1, dtype=dtype, device="cuda"))
            assert over[-1].data_ptr() not in places or side.query()          # (an allocation that waits for the device may outlast the pause)
        torch.cuda.synchronize()
        one = lambda r: r if isinstance(r, tuple) else (r,)
        assert all(torch.equal(a, b) for a, b in zip(one(got), one(want)))
