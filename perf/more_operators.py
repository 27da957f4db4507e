"""A mixture of experts in the place of a feed-forward layer, as a list of cases and a generator of more of the same ranges.

A case names one call (`op`), the type of its matrices (`dtype`) and its sizes:

    route         `k` of `experts` for each of `tokens` rows of logits: `score` "softmax" or "sigmoid", `bias` added for the choice alone,
                  `groups` of neighbouring experts of which `top_groups` are left by the sum of their `group_best` best, weights divided by
                  their sum (`renormalise`) and multiplied by `scale`; `masked`: some logits are -inf, some rows of nothing else
    route_grad    its backward pass: the gradient of the weights to that of the logits
    experts       the chosen experts' gated feed-forward layers (widths `cols` and `inner`) and their weighted sum; `save`: the projections of
                  each token's k choices are returned for the backward pass
    experts_grad  the backward pass: gradients of the tokens, of the routing weights and of the three weights
    matvec4       `tokens` products of a vector and a matrix [`rows`][`cols`] of 4-bit weights with a scale for each `group` of a row
    ffn4          gated feed-forward layer on 4-bit weights; `experts` > 0: the chosen ones' weighted sum

`pad`: columns that the rows of x (or of the logits) are apart beyond their length, as in a view of a wider matrix.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # a batch of decoders, one token each: nothing but a launch
        dict(name="route_tokens", op="route", dtype="bf16", tokens=16, experts=64, k=6, score="softmax", bias=False, groups=1, top_groups=1,
             group_best=1, renormalise=True, scale=1.0, masked=False, pad=0),
        # an ordinary training batch, balanced by a bias, experts in groups
        dict(name="route_train", op="route", dtype="fp32", tokens=16384, experts=256, k=8, score="sigmoid", bias=True, groups=8, top_groups=4,
             group_best=2, renormalise=True, scale=2.5, masked=False, pad=0),
        # odd sizes, weights that are shares of all experts
        dict(name="route_grad_odd", op="route_grad", dtype="bf16", tokens=4001, experts=60, k=4, score="softmax", renormalise=False, scale=1.0,
             masked=False, pad=3),
        # the backward pass of route_train
        dict(name="route_grad_train", op="route_grad", dtype="fp32", tokens=16384, experts=256, k=8, score="sigmoid", renormalise=True, scale=2.5,
             masked=False, pad=0),
        # a batch of decoders: the used experts' weights are read, and that is all
        dict(name="experts_decode", op="experts", dtype="bf16", tokens=16, experts=32, k=4, cols=2048, inner=1024, act="silu", save=False, pad=0),
        # a training batch, forward
        dict(name="experts_train", op="experts", dtype="bf16", tokens=8192, experts=64, k=4, cols=2048, inner=1408, act="silu", save=True, pad=0),
        # a small network's mini-batch in single precision, widths as its image-set configurations have them (784 features, 300 neurons)
        dict(name="experts_grad_fp32", op="experts_grad", dtype="fp32", tokens=500, experts=8, k=2, cols=784, inner=300, act="gelu", pad=0),
        # a training batch, backward: the largest
        dict(name="experts_grad_train", op="experts_grad", dtype="bf16", tokens=8192, experts=32, k=4, cols=2048, inner=1024, act="silu", pad=0),
        # one token of a decoder and one of its larger matrices
        dict(name="matvec4_token", op="matvec4", dtype="bf16", tokens=1, rows=8192, cols=4096, group=128, pad=0),
        # a few tokens, single precision, widths that nothing divides
        dict(name="matvec4_odd", op="matvec4", dtype="fp32", tokens=13, rows=2001, cols=1201, group=32, pad=3),
        # one token through a feed-forward layer
        dict(name="ffn4_token", op="ffn4", dtype="bf16", tokens=1, experts=0, k=1, cols=4096, inner=8192, group=128, act="silu", pad=0),
        # a batch of decoders through their experts
        dict(name="ffn4_experts", op="ffn4", dtype="fp16", tokens=8, experts=64, k=8, cols=2048, inner=1024, group=64, act="silu", pad=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width, half of them multiples of 64 where they are long enough."""
    n = _log_int(rng, lo, hi)
    return max(64, n // 64 * 64) if n >= 64 and rng.random() < 0.5 else n


def draw(rng):
    """One more case: any operator, type and direction, one to 16384 tokens, 2 to 512 experts, widths from 16 to 8192."""
    op = rng.choice(["route", "route_grad", "experts", "experts_grad", "matvec4", "ffn4"])
    case = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    act = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu", "sigmoid"])
    if op in ("route", "route_grad"):
        groups = rng.choice([1, 1, 4, 8]) if op == "route" else 1
        each = _log_int(rng, 2, 512 // groups)
        case["experts"] = groups * each
        case["tokens"] = _log_int(rng, 1, 16384)
        case["score"] = rng.choice(["softmax", "sigmoid"])
        top = rng.randint(1, groups)
        case["k"] = rng.randint(1, min(16, top * each))
        if op == "route":
            case.update(bias=rng.random() < 0.5, groups=groups, top_groups=top, group_best=rng.choice([1, 2]))
        case.update(renormalise=rng.random() < 0.5, scale=rng.choice([1.0, 1.0, 2.5]), masked=rng.random() < 0.25)
    elif op in ("experts", "experts_grad"):
        case["experts"] = _log_int(rng, 2, 128)
        case["k"] = rng.randint(1, min(8, case["experts"]))
        case["cols"] = _width(rng, 16, 4096)
        # (half a billion weights at most)
        case["inner"] = _width(rng, 16, max(16, min(4096, 500_000_000 // (3 * case["experts"] * case["cols"]))))
        most = 32768 * 2048 * 1408 // (2 if op == "experts_grad" else 1) // (16 if case["dtype"] == "fp32" else 1)
        case["tokens"] = _log_int(rng, 1, max(1, min(16384, most // (case["k"] * case["cols"] * case["inner"]))))
        case["act"] = act
        if op == "experts":
            case["save"] = rng.random() < 0.5
    else:
        case["group"] = rng.choice([32, 64, 128])
        case["tokens"] = _log_int(rng, 1, 64)
        case["cols"] = _width(rng, 16, 8192)
        if op == "matvec4":
            case["rows"] = _width(rng, 16, 16384)
        else:
            experts = rng.choice([0, _log_int(rng, 2, 128)])
            case["experts"], case["k"] = experts, rng.randint(1, min(8, experts)) if experts else 1
            case["inner"] = _width(rng, 16, max(16, min(8192, 300_000_000 // (3 * max(experts, 1) * case["cols"]))))
            case["act"] = act
    case["pad"] = rng.choice([0, 0, 0, 3, 8])
    return case


class _Inputs:
    """Random matrices of a case, in the order they are asked for."""

    def __init__(self, case, seed):
        self.type = TYPES[case["dtype"]]
        self.gen = torch.Generator(device=DEVICE)
        self.gen.manual_seed(seed)

    def normal(self, *shape, scale=1.0, pad=0, dtype=None):
        wide = (*shape[:-1], shape[-1] + pad)
        m = torch.empty(wide, device=DEVICE, dtype=dtype or self.type).normal_(0.0, scale, generator=self.gen)
        return m[..., : shape[-1]]

    def chosen(self, tokens, experts, k):
        """Indices and weights as a router gives them, some experts better liked than others."""
        z = self.normal(tokens, experts, dtype=torch.float32) + self.normal(experts, scale=0.5, dtype=torch.float32)
        top = z.topk(k, dim=1)
        return top.indices.to(torch.int32).contiguous(), top.values.softmax(1).contiguous()

    def quarters(self, *shape, group):
        """4-bit weights about their middle, and the scales of their groups."""
        q = self.normal(*shape, scale=2.6, dtype=torch.float32).add_(8).round_().clamp_(0, 15).to(torch.uint8)
        scale = self.normal(*shape[:-1], -(-shape[-1] // group), scale=0.25, dtype=torch.float32).exp_().mul_(0.4 * shape[-1] ** -0.5)
        return q, scale.to(self.type)


def prepare(case, seed):
    make = _Inputs(case, seed)
    tokens, pad, op = case["tokens"], case["pad"], case["op"]
    s = {"case": case, "seed": seed}
    if op in ("route", "route_grad"):
        experts, k = case["experts"], case["k"]
        s["logits"] = make.normal(tokens, experts, scale=1.5, pad=pad)
        if case["masked"]:
            hidden = torch.rand(tokens, experts, generator=make.gen, device=DEVICE) < 0.3
            hidden |= torch.rand(tokens, 1, generator=make.gen, device=DEVICE) < 0.02
            s["logits"][hidden] = -math.inf
        if op == "route":
            s["bias"] = make.normal(experts, scale=0.1, dtype=torch.float32) if case["bias"] else None
        else:
            s["index"] = s["logits"].float().topk(k, dim=1).indices.to(torch.int32).contiguous()
            s["dweight"] = make.normal(tokens, k, scale=0.1, dtype=torch.float32)
        return s
    s["x"] = make.normal(tokens, case["cols"], pad=pad)
    if op == "matvec4":
        s["w"] = make.quarters(case["rows"], case["cols"], group=case["group"])
    else:
        cols, inner, experts = case["cols"], case["inner"], case["experts"]
        lead = (experts,) if experts else ()
        if experts:
            s["index"], s["weight"] = make.chosen(tokens, experts, case["k"])
        for name, shape in (("w_gate", (inner, cols)), ("w_up", (inner, cols)), ("w_down", (cols, inner))):
            if op == "ffn4":
                s[name] = make.quarters(*lead, *shape, group=case["group"])
            else:
                s[name] = make.normal(*lead, *shape, scale=shape[1] ** -0.5)
        if op == "experts_grad":
            s["dy"] = make.normal(tokens, cols, scale=0.1, pad=pad)
            s["gate"], s["up"] = _projections(s)         # what the forward pass has left
    if own and op in ("matvec4", "ffn4"):
        _laid_out(s)
    return s


# ---- plain forms, in 32 bits; what decides an order in 64 -------------------------------------------------------------------------

def _scores(kind, logits):
    """softmax or sigmoid; a row of -inf alone has no scores."""
    if kind == "sigmoid":
        return 1 / (1 + (-logits).exp())
    top = logits.amax(1, keepdim=True)
    e = (logits - top.masked_fill(top == -math.inf, 0)).exp()
    total = e.sum(1, keepdim=True)
    return e / total.masked_fill(total == 0, 1)


def _first_largest(v, k):
    """Indices of the k largest of each row, in falling order, equal ones by index."""
    return v.sort(dim=1, descending=True, stable=True).indices[:, :k]


def _route(s):
    case, logits = s["case"], s["logits"].double()
    scores = _scores(case["score"], logits)
    value = scores if s["bias"] is None else scores + s["bias"].double()
    order = logits if s["bias"] is None else value
    tokens, experts = logits.shape
    if case["groups"] > 1:
        each = experts // case["groups"]
        by_order = order.view(tokens, case["groups"], each).amax(2)
        if case["group_best"] == 2:
            best = value.view(tokens, case["groups"], each).sort(dim=2, descending=True).values
            by_order = best[:, :, 0] + best[:, :, 1]
        kept = torch.zeros(tokens, case["groups"], dtype=torch.bool, device=DEVICE)
        kept.scatter_(1, _first_largest(by_order, case["top_groups"]), True)
        kept = kept.repeat_interleave(each, 1)
        # (experts of other groups behind all others, -inf included)
        index = _first_largest(order.masked_fill(~kept, math.nan).nan_to_num(nan=-1e300, neginf=-1e299), case["k"])
    else:
        index = _first_largest(order, case["k"])
    weight = scores.gather(1, index)
    if case["renormalise"]:
        total = weight.sum(1, keepdim=True)
        weight = weight / total.masked_fill(total == 0, 1)
    return index.to(torch.int32), (weight * case["scale"]).float()


def _route_grad(s):
    case, logits, index, u = s["case"], s["logits"].float(), s["index"].long(), s["dweight"] * s["case"]["scale"]
    scores = _scores(case["score"], logits)
    if case["renormalise"]:
        mine = scores.gather(1, index)
        total = mine.sum(1, keepdim=True)
        total = total.masked_fill(total == 0, math.inf)
        u = (u - (u * mine).sum(1, keepdim=True) / total) / total
    ds = torch.zeros_like(scores).scatter_add_(1, index, u)
    if case["score"] == "sigmoid":
        dlogits = ds * scores * (1 - scores)
    else:
        dlogits = scores * (ds - (ds * scores).sum(1, keepdim=True))
    return dlogits.to(s["logits"].dtype)


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


def _by_expert(index, experts):
    """For each expert that has tokens: (expert, its places in the flattened index)."""
    places = index.view(-1).sort(stable=True).indices
    counts = torch.bincount(index.view(-1), minlength=experts).tolist()
    at = 0
    for e, n in enumerate(counts):
        if n:
            yield e, places[at: at + n]
        at += n


def _projections(s):
    """x Wg^T and x Wu^T of each token's choices, a row each."""
    case, x = s["case"], s["x"].float()
    tokens, k = s["index"].shape
    gate, up = (torch.empty(tokens * k, case["inner"], dtype=s["x"].dtype, device=DEVICE) for _ in range(2))
    for e, places in _by_expert(s["index"], case["experts"]):
        rows = x[places // k]
        gate[places] = (rows @ s["w_gate"][e].float().T).to(gate.dtype)
        up[places] = (rows @ s["w_up"][e].float().T).to(up.dtype)
    return gate, up


def _experts(s):
    case, x, t = s["case"], s["x"].float(), s["x"].dtype
    tokens, k = s["index"].shape
    out = torch.empty(tokens * k, case["cols"], device=DEVICE)
    saved = [torch.empty(tokens * k, case["inner"], dtype=t, device=DEVICE) for _ in range(2 if case["save"] else 0)]
    for e, places in _by_expert(s["index"], case["experts"]):
        rows = x[places // k]
        gate, up = rows @ s["w_gate"][e].float().T, rows @ s["w_up"][e].float().T
        out[places] = (_act(case["act"], gate)[0] * up) @ s["w_down"][e].float().T
        for to, value in zip(saved, (gate, up)):
            to[places] = value.to(t)
    y = (out.view(tokens, k, -1) * s["weight"][:, :, None]).sum(1).to(t)
    return (y, *saved) if case["save"] else y


def _experts_grad(s):
    case, t = s["case"], s["x"].dtype
    x, dy, weight = s["x"].float(), s["dy"].float(), s["weight"].view(-1)
    tokens, k = s["index"].shape
    dx, dweight = torch.empty(tokens * k, case["cols"], device=DEVICE), torch.empty_like(weight)
    dw_gate, dw_up, dw_down = (torch.zeros_like(s[n]) for n in ("w_gate", "w_up", "w_down"))
    for e, places in _by_expert(s["index"], case["experts"]):
        rows, drows, w, up = x[places // k], dy[places // k], weight[places][:, None], s["up"][places].float()
        a, da = _act(case["act"], s["gate"][places].float())
        h, q = a * up, drows @ s["w_down"][e].float()
        dweight[places] = (q * h).sum(1)
        dgate, dup = w * q * up * da, w * q * a
        dx[places] = dgate @ s["w_gate"][e].float() + dup @ s["w_up"][e].float()
        dw_gate[e], dw_up[e], dw_down[e] = (dgate.T @ rows).to(t), (dup.T @ rows).to(t), ((w * drows).T @ h).to(t)
    return dx.view(tokens, k, -1).sum(1).to(t), dweight.view(tokens, k), dw_gate, dw_up, dw_down


def _values(w, group, e=None):
    """What 4-bit weights stand for."""
    q, scale = w if e is None else (w[0][e], w[1][e])
    return (q.float() - 8) * scale.float().repeat_interleave(group, -1)[..., : q.shape[-1]]


def _matvec4(s):
    return (s["x"].float() @ _values(s["w"], s["case"]["group"]).T).to(s["x"].dtype)


def _ffn4(s):
    case, x, group = s["case"], s["x"].float(), s["case"]["group"]

    def layer(rows, e):
        gate, up = rows @ _values(s["w_gate"], group, e).T, rows @ _values(s["w_up"], group, e).T
        return (_act(case["act"], gate)[0] * up) @ _values(s["w_down"], group, e).T

    if not case["experts"]:
        return layer(x, None).to(s["x"].dtype)
    tokens, k = s["index"].shape
    out = torch.empty(tokens * k, x.shape[1], device=DEVICE)
    for e, places in _by_expert(s["index"], case["experts"]):
        out[places] = layer(x[places // k], e)
    return (out.view(tokens, k, -1) * s["weight"][:, :, None]).sum(1).to(s["x"].dtype)


# ---- the calls that a user makes ----------------------------------------------------------------------------------------------

def _laid_out(s):
    """The 4-bit weights as the framework keeps them, laid out once."""
    import paper_1802_00130_b200 as gn
    for name in ("w", "w_gate", "w_up", "w_down"):
        if name in s:
            s[name + "_laid"] = gn.pack4(*s[name], group=s["case"]["group"])


def _own(s):
    import paper_1802_00130_b200 as gn
    case = s["case"]
    op = case["op"]
    if op == "route":
        return gn.route(s["logits"], case["k"], case["score"], bias=s["bias"], groups=case["groups"], top_groups=case["top_groups"],
                        group_best=case["group_best"], renormalise=case["renormalise"], scale=case["scale"])
    if op == "route_grad":
        return gn.route_grad(s["dweight"], s["logits"], s["index"], case["score"], renormalise=case["renormalise"], scale=case["scale"])
    if op == "experts":
        return gn.experts(s["x"], s["index"], s["weight"], s["w_gate"], s["w_up"], s["w_down"], case["act"], save=case["save"])
    if op == "experts_grad":
        return gn.experts_grad(s["dy"], s["x"], s["index"], s["weight"], s["gate"], s["up"], s["w_gate"], s["w_up"], s["w_down"], case["act"])
    if "w_laid" not in s and "w_gate_laid" not in s:
        _laid_out(s)
    if op == "matvec4":
        return gn.matvec4(s["x"], s["w_laid"])
    return gn.gated_ffn4(s["x"], s["w_gate_laid"], s["w_up_laid"], s["w_down_laid"], case["act"], index=s.get("index"), weight=s.get("weight"))


def run(state):
    if own:
        return _own(state)
    plain = {"route": _route, "route_grad": _route_grad, "experts": _experts, "experts_grad": _experts_grad, "matvec4": _matvec4, "ffn4": _ffn4}
    return plain[state["case"]["op"]](state)


def _used(case):
    """Experts that have a token, on average over even choices."""
    return case["experts"] * (1 - (1 - case["k"] / case["experts"]) ** case["tokens"])


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    tokens, op = case["tokens"], case["op"]
    if op in ("route", "route_grad"):
        each, chosen = tokens * case["experts"], tokens * case["k"]
        if op == "route":
            return {"bytes": each * size + 8 * chosen + (4 * case["experts"] if case["bias"] else 0), "flops": 4 * each}
        return {"bytes": 2 * each * size + 8 * chosen, "flops": 6 * each}
    cols = case["cols"]
    if op == "matvec4":
        rows = case["rows"]
        return {"bytes": rows * (-(-cols // 2) + -(-cols // case["group"]) * size) + tokens * (rows + cols) * size, "flops": 2 * tokens * rows * cols}
    inner, pairs = case["inner"], tokens * case["k"]
    choice = 8 * pairs if case["experts"] else 0
    if op == "ffn4":
        weights = 2 * inner * (-(-cols // 2) + -(-cols // case["group"]) * size) + cols * (-(-inner // 2) + -(-inner // case["group"]) * size)
        return {"bytes": int(weights * (_used(case) if case["experts"] else 1)) + 2 * tokens * cols * size + choice, "flops": 6 * pairs * cols * inner}
    weights, act = 3 * cols * inner * size, tokens * cols * size
    hidden = 2 * pairs * inner * size
    if op == "experts":
        return {"bytes": int(weights * _used(case)) + 2 * act + choice + (hidden if case["save"] else 0), "flops": 6 * pairs * cols * inner}
    return {"bytes": int(weights * _used(case)) + weights * case["experts"] + 3 * act + hidden + choice + 4 * pairs, "flops": 12 * pairs * cols * inner}


# ---- the definitions in 64 bits, as the formulas have them ------------------------------------------------------------------------

def _exact_scores(kind, z):
    if kind == "sigmoid":
        return torch.special.expit(z)
    return torch.where((z == -math.inf).all(1, keepdim=True), 0.0, torch.softmax(z, 1))


def _exact_route(s):
    """The k-th choice is the expert that k others come before: those of a kept group with a larger value, or the same and a lower number."""
    case, z = s["case"], s["logits"].double()
    tokens, experts = z.shape
    score = _exact_scores(case["score"], z)
    value = score if s["bias"] is None else score + s["bias"].double()
    order = z if s["bias"] is None else value

    def before(v):                       # [tokens][n]: how many come before each
        n = v.shape[1]
        number = torch.arange(n, device=v.device)
        ahead = torch.zeros(v.shape, dtype=torch.int64, device=v.device)
        for j in range(n):
            ahead += (v[:, j, None] > v) | ((v[:, j, None] == v) & (j < number))
        return ahead

    kept = torch.ones_like(z, dtype=torch.bool)
    groups = case["groups"]
    if groups > 1:
        each = experts // groups
        if case["group_best"] == 1:
            best = torch.stack([order[:, g * each: (g + 1) * each].amax(1) for g in range(groups)], 1)
        else:
            best = torch.stack([value[:, g * each: (g + 1) * each].topk(2, dim=1).values.sum(1) for g in range(groups)], 1)
        good = before(best) < case["top_groups"]
        kept = torch.cat([good[:, g, None].expand(tokens, each) for g in range(groups)], 1)
    rank = torch.full_like(z, experts, dtype=torch.int64)
    number = torch.arange(experts, device=z.device)
    ahead = torch.zeros_like(rank)
    for j in range(experts):
        ahead += kept[:, j, None] & ((order[:, j, None] > order) | ((order[:, j, None] == order) & (j < number)))
    rank = torch.where(kept, ahead, rank)
    index = torch.stack([(rank == j).int().argmax(1) for j in range(case["k"])], 1)
    weight = torch.take_along_dim(score, index, 1)
    if case["renormalise"]:
        weight = (weight / weight.sum(1, keepdim=True)).nan_to_num(nan=0.0)
    return index.to(torch.int32), weight * case["scale"]


def _exact_route_grad(s):
    """sum_j dw_j dw_j/dz_i, one chosen expert after the other."""
    case, z, index, dw = s["case"], s["logits"].double(), s["index"].long(), s["dweight"].double()
    score = _exact_scores(case["score"], z)
    number = torch.arange(z.shape[1], device=z.device)[None]
    ds = torch.zeros_like(z)
    chosen = torch.take_along_dim(score, index, 1)
    total = chosen.sum(1, keepdim=True) if case["renormalise"] else torch.ones_like(chosen[:, :1])
    for j in range(case["k"]):
        # w_j = scale s_j / total
        ds += case["scale"] * dw[:, j, None] * (number == index[:, j, None]) / total
        if case["renormalise"]:
            for m in range(case["k"]):
                ds -= case["scale"] * dw[:, j, None] * chosen[:, j, None] / total ** 2 * (number == index[:, m, None])
    ds = torch.where(total == 0, 0.0, ds)
    if case["score"] == "sigmoid":
        return ds * score * torch.special.expit(-z)
    return score * ds - score * torch.einsum("te,te->t", score, ds)[:, None]


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


def _exact_layers(s, weights):
    """Expert after expert, over the tokens that have chosen it; weights(name, e): its matrix."""
    case, x, index, share = s["case"], s["x"].double(), s["index"], s["weight"].double()
    y = torch.zeros_like(x)
    saved = [torch.zeros(*index.shape, case["inner"], dtype=torch.float64, device=x.device) for _ in range(2 if case.get("save") else 0)]
    for e in range(case["experts"]):
        t, j = torch.where(index == e)
        if t.numel() == 0:
            continue
        gate, up = (torch.einsum("tc,fc->tf", x[t], weights(n, e)) for n in ("w_gate", "w_up"))
        y[t] += share[t, j][:, None] * torch.einsum("tf,cf->tc", _exact_act(case["act"], gate)[0] * up, weights("w_down", e))
        for to, value in zip(saved, (gate, up)):
            to[t, j] = value
    return (y, *(m.flatten(0, 1) for m in saved)) if saved else y


def _exact_experts_grad(s):
    """From y_t = sum_j share_tj o_tj, expert after expert."""
    case, x, dy, index, share = s["case"], s["x"].double(), s["dy"].double(), s["index"], s["weight"].double()
    gate, up = (s[n].view(*index.shape, -1) for n in ("gate", "up"))
    dx, dshare = torch.zeros_like(x), torch.zeros_like(share)
    grads = [torch.zeros(s[n].shape, dtype=torch.float64, device=x.device) for n in ("w_gate", "w_up", "w_down")]
    for e in range(case["experts"]):
        t, j = torch.where(index == e)
        if t.numel() == 0:
            continue
        wg, wu, wd = (s[n][e].double() for n in ("w_gate", "w_up", "w_down"))
        a, slope = _exact_act(case["act"], gate[t, j].double())
        u = up[t, j].double()
        dshare[t, j] = torch.einsum("tc,tc->t", dy[t], torch.einsum("tf,cf->tc", a * u, wd))
        do = share[t, j][:, None] * dy[t]
        dh = torch.einsum("tc,cf->tf", do, wd)
        dgate, dup = dh * u * slope, dh * a
        dx[t] += torch.einsum("tf,fc->tc", dgate, wg) + torch.einsum("tf,fc->tc", dup, wu)
        grads[0][e], grads[1][e], grads[2][e] = (torch.einsum("tf,tc->fc", dgate, x[t]), torch.einsum("tf,tc->fc", dup, x[t]),
                                                 torch.einsum("tc,tf->cf", do, a * u))
    return (dx, dshare, *grads)


def _exact_values(w, group, e=None):
    q, scale = w if e is None else (w[0][e], w[1][e])
    column = torch.arange(q.shape[-1], device=q.device)
    return (q.double() - 8) * scale.double()[..., column // group]


def exact(case, seed):
    if work(case)["flops"] > 0.7e15:         # (about 20 seconds of 64-bit products)
        return None
    s = prepare(case, seed)
    op, group = case["op"], case.get("group")
    if op == "route":
        return _exact_route(s)
    if op == "route_grad":
        return _exact_route_grad(s)
    if op == "matvec4":
        return torch.einsum("tc,rc->tr", s["x"].double(), _exact_values(s["w"], group))
    if op == "ffn4" and not case["experts"]:
        wg, wu, wd = (_exact_values(s[n], group) for n in ("w_gate", "w_up", "w_down"))
        x = s["x"].double()
        return torch.einsum("tf,cf->tc", _exact_act(case["act"], torch.einsum("tc,fc->tf", x, wg))[0] * torch.einsum("tc,fc->tf", x, wu), wd)
    if op == "ffn4":
        return _exact_layers(s, lambda n, e: _exact_values(s[n], group, e))
    if op == "experts_grad":
        return _exact_experts_grad(s)
    return _exact_layers(s, lambda n, e: s[n][e].double())
