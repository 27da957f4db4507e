"""Plain 64-bit forms of a mixture of experts and the bounds its tests use."""
import torch

from feedforward_common import E, act64, product, rand, tiny, u, within

# an activation's FP32 value is off by a few steps: exp 2, its quotient 2, the products after it
ACT = 16 * E


def weights_of(experts, cols, inner, t, seed=0, pad=0):
    """Wg, Wu, Wd of every expert; with pad, views whose rows and experts are apart."""
    out = []
    for i, (rows, n) in enumerate(((inner, cols), (inner, cols), (cols, inner))):
        w = rand((experts * (rows + (1 if pad else 0)), n), t, seed + 10 + i, n ** -0.5, pad=pad)
        wide = w._base if pad else w
        out.append(wide.view(experts, rows + 1, n + pad)[:, :rows, :n] if pad else w.view(experts, rows, n))
    return out


def choices(tokens, experts, k, seed=0):
    """Distinct experts for each token where there are enough, unevenly liked, and their weights."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.randn(tokens, max(experts, k), generator=g, device="cuda") + torch.randn(max(experts, k), generator=g, device="cuda")
    top = z.topk(k, dim=1)
    return (top.indices % experts).to(torch.int32).contiguous(), (0.1 + torch.rand(tokens, k, generator=g, device="cuda")).contiguous()


def used(index, experts):
    """(expert, tokens, choices) of every expert that has pairs."""
    for e in range(experts):
        t, j = torch.where(index == e)
        if t.numel():
            yield e, t, j


def check_experts(got, x, index, weight, w, act, t, row=None, h_round=1.0):
    """row: rounding of a pair's row of y (none: they are FP32)."""
    row = 0.0 if row is None else row
    x64, (wg, wu, wd) = x.double(), (m.double() for m in w)
    tokens, k = index.shape
    y, y_err = torch.zeros(x.shape, dtype=torch.float64, device="cuda"), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    for e, at, j in used(index, wg.shape[0]):
        gate, gate_err = product(x64[at], wg[e], 0, 0)
        up, up_err = product(x64[at], wu[e], 0, 0)
        a, da = act64(act, gate)
        h = a * up
        h_err = up.abs() * (da.abs() + 1) * gate_err + a.abs() * up_err + (ACT * (a.abs() + gate.abs() * ACT) * up.abs()) + E * h.abs()
        o, o_err = product(h, wd[e], h_err + h_round * u(t) * h.abs() + tiny(t), 0)
        s = weight[at, j].double()[:, None]
        y.index_put_((at,), s * o, accumulate=True)
        y_err.index_put_((at,), s.abs() * (o_err + (row + (k + 2) * E) * o.abs() + tiny(t)), accumulate=True)
        if isinstance(got, tuple):
            pair = at * k + j
            within(got[1][pair], gate, gate_err + u(t) * gate.abs() + tiny(t), "gate")
            within(got[2][pair], up, up_err + u(t) * up.abs() + tiny(t), "up")
    within(got[0] if isinstance(got, tuple) else got, y, y_err + u(t) * y.abs() + tiny(t), "y")


def check_experts_grad(got, dy, x, index, weight, gate, up, w, act, t):
    tokens, k = index.shape
    dy64, x64, (wg, wu, wd) = dy.double(), x.double(), (m.double() for m in w)
    new = lambda like: torch.zeros(like.shape, dtype=torch.float64, device="cuda")
    dx, dx_err, ds, ds_err = new(x), new(x), new(weight), new(weight)
    grads, errs = [new(m) for m in w], [new(m) for m in w]
    rel = u(t) + 3 * E
    for e, at, j in used(index, wg.shape[0]):
        pair, s = at * k + j, weight[at, j].double()[:, None]
        g64, u64, d = gate[pair].double(), up[pair].double(), dy64[at]
        a, da = act64(act, g64)
        slack = ACT * (a.abs() + g64.abs() * ACT)
        q, q_err = product(d, wd[e].T, 0, 0)
        h = a * u64
        # a sum of `inner` products, in FP32 pieces of 64 columns and sums of those: errors of a piece's additions, as product's, and of its terms
        ds[at, j] = (q * h).sum(1)
        spread = ((q * h) ** 2).sum(1).sqrt()
        ds_err[at, j] = ((q_err * h.abs()) ** 2).sum(1).sqrt() * 7 + ((q.abs() * slack * u64.abs()).sum(1)) + 7 * E * 2 * (64 + h.shape[1] / 64) ** 0.5 * 7 * spread + 80 * E * ds[at, j].abs()
        h_s, dgate, dup = s * h, s * q * u64 * da, s * q * a
        h_err = rel * h_s.abs() + tiny(t) + s * slack * u64.abs()
        dgate_err = s * q_err * (u64 * da).abs() + rel * dgate.abs() + tiny(t) + (s * q * u64).abs() * ACT * 2
        dup_err = s * q_err * a.abs() + rel * dup.abs() + tiny(t) + slack * (s * q).abs()
        both, both_err = product(torch.cat([dgate, dup], 1), torch.cat([wg[e], wu[e]], 0).T, torch.cat([dgate_err, dup_err], 1), 0)
        dx.index_put_((at,), both, accumulate=True)
        dx_err.index_put_((at,), both_err + (k + 2) * E * both.abs(), accumulate=True)
        xs = x64[at]
        for i, (ref, err) in enumerate((product(dgate.T, xs.T, dgate_err.T, 0), product(dup.T, xs.T, dup_err.T, 0), product(d.T, h_s.T, 0, h_err.T))):
            grads[i][e], errs[i][e] = ref, err
    within(got[0], dx, dx_err + u(t) * dx.abs() + tiny(t), "dx")
    within(got[1], ds, ds_err + E * ds.abs() + 1e-37, "dweight")
    for g, ref, err, name in zip(got[2:], grads, errs, ("dw_gate", "dw_up", "dw_down")):
        within(g, ref, err + u(t) * ref.abs() + tiny(t), name)
