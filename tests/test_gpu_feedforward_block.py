"""The feed-forward block's operators together, as a training step and a decoder use them: out = x + dropout(ffn(norm(x)))."""
import threading

import pytest
import torch

import paper_1802_00130_b200 as gn
from feedforward_common import TYPES, act64, mask_of, rand, vec

pytestmark = pytest.mark.gpu

P, KEY, STEP = 0.2, 77, 5


def parameters(cols, inner, t):
    return dict(w=vec(cols, t, 1, 0.1, 1.0), b=vec(cols, t, 2, 0.1), gate=rand((inner, cols), t, 3, cols ** -0.5), up=rand((inner, cols), t, 4, cols ** -0.5),
                down=rand((cols, inner), t, 5, inner ** -0.5))


def forward(x, q, stream=None, step=STEP, device_step=None):
    h, mean, rstd = gn.layer_norm(x, q["w"], q["b"], save=True, stream=stream)
    y, gate, up = gn.gated_ffn(h, q["gate"], q["up"], q["down"], save=True, stream=stream)
    return gn.dropout(y, P, KEY, step, residual=x, device_step=device_step, stream=stream), (h, mean, rstd, gate, up)


def backward(dout, x, q, kept, stream=None, step=STEP, device_step=None):
    h, mean, rstd, gate, up = kept
    dy = gn.dropout(dout, P, KEY, step, device_step=device_step, stream=stream)
    dh, *dw = gn.gated_ffn_grad(dy, h, gate, up, q["gate"], q["up"], q["down"], stream=stream)
    dx, dnw, dnb = gn.layer_norm_grad(dh, x, mean, rstd, q["w"], add=dout, stream=stream)
    return [dx, dnw, dnb, *dw]


def block64(x, q, keep):
    d = x - x.mean(1, keepdim=True)
    h = d * (d.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * q["w"] + q["b"]
    return x + torch.where(keep, ((act64("silu", h @ q["gate"].T)[0] * (h @ q["up"].T)) @ q["down"].T) / (1 - P), 0.0)


@pytest.mark.parametrize("rows,cols,inner", [(1, 64, 96), (40, 129, 77), (300, 256, 520), (1000, 520, 1032)])
@pytest.mark.parametrize("t", TYPES)
def test_block_and_its_gradients(t, rows, cols, inner):
    """Against automatic differentiation of the 64-bit form.

    Each value of the block has at most five roundings to the type behind it (norm, projection or h, y, sum, and dy, dh, dgate in the
    backward pass), independent and of at most u each: in the 2-norm they stay below 5 u of the result times the gain of what follows, about one here."""
    t = TYPES[t]
    q, x, dout = parameters(cols, inner, t), rand((rows, cols), t, 6), rand((rows, cols), t, 7)
    out, kept = forward(x, q)
    got = backward(dout, x, q, kept)
    leaves = [x.double().requires_grad_()] + [q[k].double().requires_grad_() for k in ("w", "b", "gate", "up", "down")]
    ref = block64(leaves[0], dict(zip(("w", "b", "gate", "up", "down"), leaves[1:])), mask_of((rows, cols), P, KEY, STEP))
    grads = torch.autograd.grad(ref, leaves, dout.double())
    limit = 5 * torch.finfo(t).eps / 2 if t != torch.float32 else 2e-6
    for g, r, name in zip([out] + got, (ref.detach(), *grads), ("out", "dx", "dnorm_w", "dnorm_b", "dw_gate", "dw_up", "dw_down")):
        off = float((g.double() - r).norm() / r.norm())
        assert off < limit, (name, off)


def test_other_streams_and_two_at_once():
    """The block on two streams at the same time, from two threads, gives what it gives alone."""
    t = torch.bfloat16
    q = parameters(256, 520, t)
    xs, douts = [rand((400, 256), t, s) for s in (1, 2)], [rand((400, 256), t, s) for s in (3, 4)]
    want = []
    for x, d in zip(xs, douts):
        out, kept = forward(x, q)
        want.append([out] + backward(d, x, q, kept))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]

    def work(k):
        for _ in range(20):
            out, kept = forward(xs[k], q, stream=streams[k])
            got[k] = [out] + backward(douts[k], xs[k], q, kept, stream=streams[k])

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    [th.start() for th in threads]
    [th.join() for th in threads]
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[k], want[k]))


@pytest.mark.parametrize("t", TYPES)
def test_captured_training_step(t):
    """Two graphs of the same step on different inputs, replayed in turn and at once, against eager calls."""
    t = TYPES[t]
    q = parameters(264, 392, t)
    xs, dout = [rand((300, 264), t, s) for s in (1, 2)], rand((300, 264), t, 3)
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    forward(xs[0], q)
    graphs, outs = [], []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out, kept = forward(x, q, device_step=counter)
            outs.append([out] + backward(dout, x, q, kept, device_step=counter))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(3):
        counter.fill_(k)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for x, got in zip(xs, outs):
            out, kept = forward(x, q, step=STEP + k)
            assert all(torch.equal(a, b) for a, b in zip(got, [out] + backward(dout, x, q, kept, step=STEP + k)))


def test_single_tokens_agree_with_a_batch():
    """A decoder's calls, one token each, and the batch of them: both within the type's rounding of the 64-bit form, so of one another."""
    t = torch.bfloat16
    q, x = parameters(512, 1032, t), rand((200, 512), t, 8)
    h = gn.layer_norm(x, q["w"], q["b"])
    batch = gn.gated_ffn(h, q["gate"], q["up"], q["down"])
    for n in (1, 2, 5, 9, 17, 33):
        some = gn.gated_ffn(gn.layer_norm(x[:n], q["w"], q["b"]), q["gate"], q["up"], q["down"])
        # h and y rounded once in each form: four half steps at most, independent
        assert float((some.double() - batch[:n].double()).norm() / batch[:n].double().norm()) < 4 * torch.finfo(t).eps / 2


@pytest.mark.parametrize("rows", [3, 300])
def test_arguments_dropped_after_a_call_on_another_stream(rows):
    """Their memory is not handed out again before that stream has read it: the calls wait behind a pause of some 50 ms, while the current
    stream allocates tensors of the same sizes and fills them."""
    t = torch.bfloat16
    q, side = parameters(256, 520, t), torch.cuda.Stream()
    x, dout = rand((rows, 256), t, 1), rand((rows, 256), t, 2)
    step = torch.tensor([1], dtype=torch.int64, device="cuda")
    h, mean, rstd = gn.layer_norm(x, q["w"], q["b"], save=True)
    y, gate, up = gn.gated_ffn(h, q["gate"], q["up"], q["down"], save=True)
    W = (q["gate"], q["up"], q["down"])
    calls = [(gn.layer_norm, (x, q["w"], q["b"])), (gn.layer_norm_grad, (dout, x, mean, rstd, q["w"], dout)), (gn.dropout, (x, P, KEY, STEP, dout, step)),
             (gn.gated_ffn, (h, *W)), (gn.gated_ffn_grad, (dout, h, gate, up, *W))]
    for call, args in calls:
        want = call(*args)
        mine = [a.clone() if torch.is_tensor(a) else a for a in args]
        places = {a.data_ptr(): a.shape for a in mine if torch.is_tensor(a)}
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        got = call(*mine, stream=side)
        del mine
        over = []
        for shape in [shape for shape in places.values() for _ in range(4)]:
            over.append(torch.full(shape, 1 if tuple(shape) == (1,) else 7, dtype=torch.int64 if tuple(shape) == (1,) else t, device="cuda"))
            assert over[-1].data_ptr() not in places or side.query()          # (an allocation that waits for the device may outlast the pause)
        torch.cuda.synchronize()
        one = lambda r: r if isinstance(r, tuple) else (r,)
        assert all(torch.equal(a, b) for a, b in zip(one(got), one(want)))


def test_captured_on_a_given_stream():
    """The block's calls on the stream that captures, given by name, with arguments that are dropped meanwhile."""
    t = torch.bfloat16
    q, x, dout, side = parameters(256, 520, t), rand((300, 256), t, 1), rand((300, 256), t, 2), torch.cuda.Stream()
    out, kept = forward(x, q)
    want = [out] + backward(dout, x, q, kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, kept = forward(x, q, stream=side)
        got = [out] + backward(dout, x, q, kept, stream=side)
        del kept
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_stream_is_a_stream_of_the_tensors_device():
    x = rand((4, 16), torch.bfloat16, 1)
    side, want = torch.Stream(device="cuda"), gn.layer_norm(x)
    torch.cuda.synchronize()
    got = gn.layer_norm(x, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    for bad in (0, "side", torch.device("cuda")):
        with pytest.raises(TypeError, match="torch.cuda.Stream"):
            gn.layer_norm(x, stream=bad)
