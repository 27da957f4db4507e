"""The feed-forward operators of a language model's block, as a list of cases and a generator of more of the same ranges.

A case names one call (`op`), the type of its matrices (`dtype`) and its sizes:

    norm          layer norm of `rows` x `cols`, with the rows' means and reciprocal standard deviations (training) or
                  without (`save` false)
    norm_grad     its backward pass: gradients of the rows, the weight and the bias; `add`: the gradient that reaches the rows
                  past the norm, over the residual path, is added to theirs
    dropout       dropout by a counter-based generator; `residual`: added to what is left (the end of a block)
    ffn           gated feed-forward block  y = (act(x Wg^T) * (x Wu^T)) Wd^T  of `rows` tokens, widths `cols` and `inner`;
                  `save`: the two projections are returned for the backward pass
    ffn_grad      its backward pass: gradients of x and of the three weights

`pad`: columns that the rows of x (or of dy) are apart beyond their length, as in a view of a wider matrix.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # one token of a decoder: nothing but a launch
        dict(name="norm_token", op="norm", dtype="bf16", rows=1, cols=4096, save=False, pad=0),
        # an ordinary training batch of a wide model
        dict(name="norm_train", op="norm", dtype="bf16", rows=16384, cols=4096, save=True, pad=0),
        # features after a selection, single precision, odd everything
        dict(name="norm_grad_odd", op="norm_grad", dtype="fp32", rows=4001, cols=1201, add=False, pad=0),
        # the backward pass of norm_train, with the residual path's gradient
        dict(name="norm_grad_train", op="norm_grad", dtype="bf16", rows=16384, cols=4096, add=True, pad=0),
        # hidden activations of a small network's mini-batch
        dict(name="dropout_small", op="dropout", dtype="fp32", rows=131, cols=617, p=0.5, residual=False, pad=0),
        # the end of a block in training: dropout and residual addition; its backward pass is the same without the residual
        dict(name="dropout_train", op="dropout", dtype="bf16", rows=16384, cols=4096, p=0.1, residual=True, pad=0),
        # one token of a decoder: the weights are read, and that is all
        dict(name="ffn_token", op="ffn", dtype="bf16", rows=1, cols=4096, inner=8192, act="silu", save=False, pad=0),
        # a batch of decoders, one token each
        dict(name="ffn_batch", op="ffn", dtype="fp16", rows=48, cols=2048, inner=8192, act="gelu", save=False, pad=0),
        # a training batch, forward
        dict(name="ffn_train", op="ffn", dtype="bf16", rows=8192, cols=4096, inner=8192, act="silu", save=True, pad=0),
        # a small network in single precision, as its image-set configurations have it (784 features, 2000 neurons)
        dict(name="ffn_grad_fp32", op="ffn_grad", dtype="fp32", rows=3000, cols=784, inner=2000, act="sigmoid", pad=0),
        # widths that no tile and no 16-byte row divides
        dict(name="ffn_grad_odd", op="ffn_grad", dtype="fp16", rows=1003, cols=617, inner=1201, act="gelu_tanh", pad=0),
        # a training batch, backward: the largest
        dict(name="ffn_grad_train", op="ffn_grad", dtype="bf16", rows=8192, cols=4096, inner=8192, act="silu", pad=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width, half of them multiples of 64 where they are long enough."""
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if n >= 64 and rng.random() < 0.5 else n


def draw(rng):
    """One more case: any operator, type and direction, one to 65536 rows, widths from 8 to 16384."""
    op = rng.choice(["norm", "norm_grad", "dropout", "ffn", "ffn", "ffn_grad"])
    case = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    pad = rng.choice([0, 0, 0, 3, 8])
    if op in ("norm", "norm_grad", "dropout"):
        case["cols"] = _width(rng, 8, 16384)
        case["rows"] = _log_int(rng, 1, max(1, min(65536, 16384 * 4096 // (case["cols"] + 8))))
        if op == "norm":
            case["save"] = rng.random() < 0.5
        elif op == "norm_grad":
            case["add"] = rng.random() < 0.5
        else:
            case.update(p=rng.choice([0.0, 0.05, 0.1, 0.25, 0.5, 0.9]), residual=rng.random() < 0.5)
    else:
        most = 8192 * 4096 * 8192 // (8 if case["dtype"] == "fp32" else 1)
        case["cols"], case["inner"] = _width(rng, 16, 8192), _width(rng, 16, 16384)
        case["rows"] = _log_int(rng, 1, max(1, min(16384, most // (case["cols"] * case["inner"]))))
        case["act"] = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu", "sigmoid"])
        if op == "ffn":
            case["save"] = rng.random() < 0.5
    case["pad"] = pad
    return case


class _Inputs:
    """Random matrices of a case, in the order they are asked for."""

    def __init__(self, case, seed):
        self.type = TYPES[case["dtype"]]
        self.gen = torch.Generator(device=DEVICE)
        self.gen.manual_seed(seed)

    def normal(self, rows, cols, scale=1.0, shift=0.0, pad=0):
        m = torch.randn(rows, cols + pad, generator=self.gen, device=DEVICE).mul_(scale).add_(shift)
        return m.to(self.type)[:, :cols]

    def vector(self, n, scale=1.0, shift=0.0):
        return torch.randn(n, generator=self.gen, device=DEVICE).mul_(scale).add_(shift).to(self.type)


def prepare(case, seed):
    make = _Inputs(case, seed)
    rows, cols, pad = case["rows"], case["cols"], case["pad"]
    s = {"case": case, "seed": seed}
    if case["op"] in ("norm", "norm_grad"):
        # activations of a residual path: spread about a mean that is not zero, some channels larger than the others
        s["x"] = make.normal(rows, cols, 1.5, 0.25, pad)
        s["x"][:, ::61] *= 4
        s["weight"], s["bias"] = make.vector(cols, 0.1, 1.0), make.vector(cols, 0.1)
        if case["op"] == "norm_grad":
            s["dy"] = make.normal(rows, cols, 0.1, 0.0, pad)
            s["add"] = make.normal(rows, cols, 0.1) if case["add"] else None
            x = s["x"].float()                     # what the forward pass has left
            mean = x.mean(1, keepdim=True)
            s["mean"], s["rstd"] = mean[:, 0].contiguous(), ((x - mean).square().mean(1) + EPS).rsqrt()
    elif case["op"] == "dropout":
        s["x"] = make.normal(rows, cols, 1.0, 0.0, pad)
        s["residual"] = make.normal(rows, cols, 2.0) if case["residual"] else None
        s["key"], s["step"] = seed * 0x9E3779B1 + 12345, 7
    else:
        inner = case["inner"]
        s["x"] = make.normal(rows, cols, 1.0, 0.0, pad)
        s["w_gate"] = make.normal(inner, cols, cols ** -0.5)
        s["w_up"] = make.normal(inner, cols, cols ** -0.5)
        s["w_down"] = make.normal(cols, inner, inner ** -0.5)
        if case["op"] == "ffn_grad":
            s["dy"] = make.normal(rows, cols, 0.1, 0.0, pad)
            s["gate"] = (s["x"].float() @ s["w_gate"].float().T).to(make.type)     # what the forward pass has left
            s["up"] = (s["x"].float() @ s["w_up"].float().T).to(make.type)
    return s


# ---- plain forms, in 32 bits --------------------------------------------------------------------------------------------------

def _norm(s):
    x, t = s["x"].float(), s["x"].dtype
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = (d.square().mean(1, keepdim=True) + EPS).rsqrt()
    y = (d * rstd * s["weight"].float() + s["bias"].float()).to(t)
    return (y, mean[:, 0], rstd[:, 0]) if s["case"]["save"] else y


def _norm_grad(s):
    x, dy, t = s["x"].float(), s["dy"].float(), s["x"].dtype
    rstd = s["rstd"][:, None]
    xhat = (x - s["mean"][:, None]) * rstd
    g = dy * s["weight"].float()
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if s["add"] is not None:
        dx = dx + s["add"].float()
    return dx.to(t), (dy * xhat).sum(0).to(t), dy.sum(0).to(t)


_LOW = 0xFFFFFFFF


def _philox_round(c, key):
    """One round of Philox4x32 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) on 32-bit words
    held in 64 bits; a product keeps its 64 bits through the wrap-around of the signed type."""
    a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
    return [((b >> 32) & _LOW) ^ c[1] ^ key[0], b & _LOW, ((a >> 32) & _LOW) ^ c[3] ^ key[1], a & _LOW]


def _dropout(s):
    x, p, t = s["x"], s["case"]["p"], s["x"].dtype
    rows, cols = x.shape
    block = torch.arange((rows * cols + 3) // 4, device=x.device)
    step = torch.full_like(block, s["step"])
    c = [block & _LOW, block >> 32, step & _LOW, step >> 32]
    key = (s["key"] & _LOW, s["key"] >> 32 & _LOW)
    for k in range(10):                            # the rounds depend on one another
        c = _philox_round(c, ((key[0] + k * 0x9E3779B9) & _LOW, (key[1] + k * 0xBB67AE85) & _LOW))
    words = torch.stack(c, 1).view(-1)[: rows * cols].view(rows, cols)
    keep = words >= round(p * 2 ** 32)
    y = torch.where(keep, x.float() * (1 / (1 - p)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(t)


def _act(name, v):
    """The activation and its derivative."""
    if name == "relu":
        return v.clamp(min=0), (v > 0).to(v.dtype)
    if name in ("sigmoid", "silu"):
        z = 1 / (1 + (-v).exp())
        return (z, z * (1 - z)) if name == "sigmoid" else (v * z, z * (1 + v * (1 - z)))
    if name == "gelu":
        cdf = 0.5 * (1 + (v * 0.5 ** 0.5).erf())
        return v * cdf, cdf + v * (-0.5 * v * v).exp() * (2 * math.pi) ** -0.5
    k = (2 / math.pi) ** 0.5
    th = (k * (v + 0.044715 * v * v * v)).tanh()
    return 0.5 * v * (1 + th), 0.5 * (1 + th) + 0.5 * v * (1 - th * th) * k * (1 + 3 * 0.044715 * v * v)


def _ffn(s):
    x, t = s["x"].float(), s["x"].dtype
    gate, up = x @ s["w_gate"].float().T, x @ s["w_up"].float().T
    y = ((_act(s["case"]["act"], gate)[0] * up) @ s["w_down"].float().T).to(t)
    return (y, gate.to(t), up.to(t)) if s["case"]["save"] else y


def _ffn_grad(s):
    x, dy, t = s["x"].float(), s["dy"].float(), s["x"].dtype
    up = s["up"].float()
    a, da = _act(s["case"]["act"], s["gate"].float())
    dh = dy @ s["w_down"].float()
    dup, dgate = dh * a, dh * up * da
    dx = dgate @ s["w_gate"].float() + dup @ s["w_up"].float()
    return dx.to(t), (dgate.T @ x).to(t), (dup.T @ x).to(t), (dy.T @ (a * up)).to(t)


# ---- the calls that a user makes ----------------------------------------------------------------------------------------------

def _own(s):
    import paper_1802_00130_b200 as gn
    case = s["case"]
    if case["op"] == "norm":
        return gn.layer_norm(s["x"], s["weight"], s["bias"], EPS, save=case["save"])
    if case["op"] == "norm_grad":
        return gn.layer_norm_grad(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], add=s["add"])
    if case["op"] == "dropout":
        return gn.dropout(s["x"], case["p"], s["key"], step=s["step"], residual=s["residual"])
    if case["op"] == "ffn":
        return gn.gated_ffn(s["x"], s["w_gate"], s["w_up"], s["w_down"], case["act"], save=case["save"])
    return gn.gated_ffn_grad(s["dy"], s["x"], s["gate"], s["up"], s["w_gate"], s["w_up"], s["w_down"], case["act"])


def run(state):
    if own:
        return _own(state)
    plain = {"norm": _norm, "norm_grad": _norm_grad, "dropout": _dropout, "ffn": _ffn, "ffn_grad": _ffn_grad}
    return plain[state["case"]["op"]](state)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    rows, cols = case["rows"], case["cols"]
    each = rows * cols
    if case["op"] == "norm":
        return {"bytes": (2 * each + 2 * cols) * size + (8 * rows if case["save"] else 0), "flops": 8 * each}
    if case["op"] == "norm_grad":
        return {"bytes": ((4 if case["add"] else 3) * each + 3 * cols) * size + 8 * rows, "flops": 14 * each}
    if case["op"] == "dropout":
        return {"bytes": (3 if case["residual"] else 2) * each * size, "flops": 2 * each}
    inner = case["inner"]
    weights, hidden = 3 * cols * inner, rows * inner
    if case["op"] == "ffn":
        return {"bytes": (weights + 2 * each + (2 * hidden if case["save"] else 0)) * size, "flops": 6 * each * inner}
    return {"bytes": (2 * weights + 3 * each + 2 * hidden) * size, "flops": 12 * each * inner}


# ---- the definitions in 64 bits, element by element as the formulas have them ---------------------------------------------------

def _exact_norm(s):
    x = s["x"].double()
    n = x.shape[1]
    mean = torch.einsum("rc->r", x) / n
    var = torch.einsum("rc,rc->r", x - mean[:, None], x - mean[:, None]) / n
    y = (x - mean[:, None]) / torch.sqrt(var + EPS)[:, None] * s["weight"].double()[None] + s["bias"].double()[None]
    return (y, mean, 1 / torch.sqrt(var + EPS)) if s["case"]["save"] else y


def _exact_norm_grad(s):
    """dx_i = sum_j dL/dxhat_j dxhat_j/dx_i with dxhat_j/dx_i = rstd (delta_ij - (1 + xhat_i xhat_j) / n)."""
    x, dy, w = s["x"].double(), s["dy"].double(), s["weight"].double()
    n = x.shape[1]
    rstd = s["rstd"].double()
    xhat = (x - s["mean"].double()[:, None]) * rstd[:, None]
    along, across = torch.einsum("rc,c->r", dy, w), torch.einsum("rc,c,rc->r", dy, w, xhat)
    dx = rstd[:, None] * (dy * w - (along[:, None] + xhat * across[:, None]) / n)
    if s["add"] is not None:
        dx += s["add"].double()
    return dx, torch.einsum("rc,rc->c", dy, xhat), torch.einsum("rc->c", dy)


def _mul32(a, m):
    """High and low words of the product of 32-bit words and a constant, by halves of 16 bits."""
    al, ah, ml, mh = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
    low, mid = al * ml, ah * ml + ((al * ml) >> 16)
    mid2 = al * mh + (mid & 0xFFFF)
    return ah * mh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)


def _exact_dropout(s):
    x, p = s["x"], s["case"]["p"]
    n = x.numel()
    i = torch.arange(-(-n // 4), device=x.device, dtype=torch.int64)
    w = {0: i % 2 ** 32, 1: i // 2 ** 32, 2: torch.full_like(i, s["step"] % 2 ** 32), 3: torch.full_like(i, s["step"] // 2 ** 32)}
    k0, k1 = s["key"] % 2 ** 32, s["key"] // 2 ** 32 % 2 ** 32
    for _ in range(10):
        h0, l0 = _mul32(w[0], 0xD2511F53)
        h1, l1 = _mul32(w[2], 0xCD9E8D57)
        w = {0: h1 ^ w[1] ^ k0, 1: l1, 2: h0 ^ w[3] ^ k1, 3: l0}
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    word = torch.empty(4 * i.numel(), device=x.device, dtype=torch.int64)
    for k in range(4):
        word[k::4] = w[k]
    y = x.double() / (1 - p)
    y[(word[:n] < round(p * 2 ** 32)).view_as(y)] = 0
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_act(name, v):
    z = torch.special.expit(v)
    if name == "relu":
        return torch.where(v > 0, v, 0.0), torch.where(v > 0, 1.0, 0.0).to(v.dtype)
    if name == "sigmoid":
        return z, z * torch.special.expit(-v)
    if name == "silu":
        return v * z, z + v * z * torch.special.expit(-v)
    if name == "gelu":
        cdf = torch.special.ndtr(v)
        return v * cdf, cdf + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    # 0.5 (1 + tanh q) = 1 / (1 + exp(-2 q))
    q = math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
    c = torch.special.expit(2 * q)
    return v * c, c + 2 * v * c * torch.special.expit(-2 * q) * math.sqrt(2 / math.pi) * (1 + 0.134145 * v ** 2)


def _exact_ffn(s):
    x, wg, wu, wd = (s[k].double() for k in ("x", "w_gate", "w_up", "w_down"))
    gate, up = torch.einsum("tc,fc->tf", x, wg), torch.einsum("tc,fc->tf", x, wu)
    y = torch.einsum("tf,cf->tc", _exact_act(s["case"]["act"], gate)[0] * up, wd)
    return (y, gate, up) if s["case"]["save"] else y


def _exact_ffn_grad(s):
    x, dy, gate, up, wg, wu, wd = (s[k].double() for k in ("x", "dy", "gate", "up", "w_gate", "w_up", "w_down"))
    a, slope = _exact_act(s["case"]["act"], gate)
    dh = torch.einsum("tc,cf->tf", dy, wd)
    dgate, dup = dh * up * slope, dh * a
    dx = torch.einsum("tf,fc->tc", dgate, wg) + torch.einsum("tf,fc->tc", dup, wu)
    return dx, torch.einsum("tf,tc->fc", dgate, x), torch.einsum("tf,tc->fc", dup, x), torch.einsum("tc,tf->cf", dy, a * up)


def exact(case, seed):
    s = prepare(case, seed)
    forms = {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "dropout": _exact_dropout, "ffn": _exact_ffn,
             "ffn_grad": _exact_ffn_grad}
    return forms[case["op"]](s)
