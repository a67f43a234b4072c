"""Measured cases of the mixture-of-experts operators: routing, the experts' products and the token embedding.

A case names one of four passes:
  route   T x E router logits to k experts a token (weights, experts and the rows in expert order); with `train`
          also the gradient of the logits
  up      the first product of an expert, x (T, n) to rows (T k, m): "fwd", or "bwd" (gradients of x and W)
  down    the second product and the weighted sum back to tokens, h (T k, n) to (T, m): "fwd", or "bwd" (gradients of
          h, W and the routing weights)
  embed   the embedding lookup of T tokens in a V x D table with a scale; with `train` also the table's gradient
Fields: T tokens, E experts, k experts a token, n x m the weight of one expert; score, bias, groups, top, pair (a group
counts its two highest scores), renorm, scale, pad (share of tokens without experts or without an id), dtype.
"""
import math

import torch

own = False

F32, BF16 = "float32", "bfloat16"
ROUTE = dict(kind="route", E=128, k=2, score="softmax", bias=False, groups=1, top=1, pair=False, renorm=True, scale=1.0,
             pad=0.0, dtype=F32, train=True)
MATS = dict(E=128, k=2, pad=0.0, dtype=BF16)
EMBED = dict(kind="embed", V=50304, D=2048, scale=1.0, pad=0.0, dtype=BF16, train=True)


def listed():
    def case(base, name, **kw):
        return dict(base, name=name, **kw)

    return [
        # one token of a model that answers: 2 of 128 experts, launches and latency
        case(ROUTE, "route_one_token", T=1, train=False),
        # a training step's 8192 tokens over the benchmark model's 128 experts
        case(ROUTE, "route_step", T=8192),
        # balanced routing inside groups of experts, bf16 logits, an odd number of tokens, padded ones among them
        case(ROUTE, "route_groups", T=40001, E=192, k=6, score="sigmoid", bias=True, groups=6, top=3, pair=True,
             scale=1.5, pad=0.03, dtype=BF16),
        # one token through the first expert product: two experts' weights have to be read, nothing else counts
        case(MATS, "up_one_token", kind="up", T=1, n=2048, m=8192, dir="fwd"),
        # the tiny model's backward pass over a short odd batch: launches and latency
        case(MATS, "up_tiny_backward", kind="up", T=251, E=8, n=256, m=1024, dir="bwd"),
        # a micro-batch of 1024 tokens over all 128 experts: 16 rows an expert, bound by the weights' bytes
        case(MATS, "up_micro_batch", kind="up", T=1024, n=2048, m=8192, dir="fwd"),
        # a quarter of the experts with 128 rows each, as in a step of 8192 tokens: gradients of the down projection
        case(MATS, "down_step_backward", kind="down", T=2048, E=32, n=8192, m=2048, dir="bwd"),
        # widths that are no multiple of 8 and a ragged number of rows, some tokens without experts
        case(MATS, "down_odd", kind="down", T=3001, E=16, k=3, n=2765, m=1031, pad=0.05, dir="fwd"),
        # wide experts with about 2000 rows each: bound by the matrix cores
        case(MATS, "up_wide", kind="up", T=8192, E=8, n=4096, m=11008, dir="fwd"),
        # a few new tokens in bf16: latency
        case(EMBED, "embed_few_tokens", T=16, train=False),
        # a training step's tokens: rows of the table's gradient without tokens are most of its bytes
        case(EMBED, "embed_step", T=8192),
        # a long batch on a float32 table of odd width: frequent tokens hold thousands of rows
        case(EMBED, "embed_long_odd", T=65537, V=32003, D=1031, scale=32.0, pad=0.02, dtype=F32),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):
        n = log(lo, hi)
        return n if rng.random() < 0.4 else max(lo, n // 64 * 64)

    kind = rng.choice(("route", "route", "up", "up", "down", "down", "embed", "embed"))
    pad = rng.choice((0.0, 0.0, 0.05))
    if kind == "route":
        groups = rng.choice((1, 1, 4, 6))
        E = groups * log(8 if groups == 1 else 4, 192 // groups)
        top = rng.randrange(1, groups + 1)
        bias = rng.random() < 0.5
        return dict(ROUTE, T=log(1, 40000), E=E, k=min(rng.choice((1, 2, 2, 4, 6, 8)), top * (E // groups)),
                    score=rng.choice(("softmax", "sigmoid")), bias=bias, groups=groups, top=top,
                    pair=bias and groups > 1 and rng.random() < 0.5, renorm=rng.random() < 0.7,
                    scale=rng.choice((1.0, 1.5)), pad=pad, dtype=rng.choice((F32, BF16)), train=rng.random() < 0.7)
    if kind == "embed":
        while True:
            c = dict(EMBED, T=log(1, 65537), V=log(300, 60000), D=width(64, 4096), scale=rng.choice((1.0, 1.0, 45.25)),
                     pad=pad, dtype=rng.choice((F32, BF16, BF16)), train=rng.random() < 0.7)
            if work(c)["bytes"] <= 4e8:
                return c
    while True:
        E = log(4, 128)
        c = dict(MATS, kind=kind, T=log(1, 8192), E=E, k=min(E, rng.choice((1, 2, 2, 4))), n=width(64, 8192),
                 m=width(64, 8192), pad=pad, dir=rng.choice(("fwd", "bwd")))
        w = work(c)
        if c["E"] * c["n"] * c["m"] <= 540_000_000 and w["flops"] <= 1.4e12:
            return c


# ---- inputs -----------------------------------------------------------------------------------
def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + k) & (2**62 - 1))
    return g


def _logits(c, gen):
    """Router logits: each expert's popularity (its logarithm; the shares are exponential) and a token's own part."""
    share = torch.rand(c["E"], generator=gen, device="cuda").clamp_(min=1e-3).log_().neg_().clamp_(min=1e-2).log_()
    noise = torch.rand((c["T"], c["E"]), generator=gen, device="cuda").clamp_(min=1e-9)
    return share - noise.log_().neg_().clamp_(min=1e-9).log_()   # share + Gumbel noise


def _none(c, gen):
    """Which tokens are padding."""
    return torch.rand(c["T"], generator=gen, device="cuda") < c["pad"]


def _decided(c, logits, bias):
    """Rows of logits whose choice 32 bits cannot decide (two scores, or two groups, closer than 1e-5 without being
    equal: one token in some thousands) take the logits of another token: the choice is a whole number that has to be
    the same however the scores are rounded. Choices by the logits themselves are exact and need none of this."""
    if bias is None:
        return logits
    x = logits.double()
    s = torch.softmax(x, -1) if c["score"] == "softmax" else torch.sigmoid(x)
    v = s + bias.double()
    per = c["E"] // c["groups"]
    by = v.view(-1, c["groups"], per).sort(-1, descending=True).values
    g = by[..., :2 if c["pair"] else 1].sum(-1)
    gs, gi = g.sort(-1, descending=True)
    close = torch.zeros(c["T"], dtype=torch.bool, device="cuda")
    if c["top"] < c["groups"]:
        close |= gs[:, c["top"] - 1] - gs[:, c["top"]] < 1e-5
    kept = torch.zeros_like(g, dtype=torch.bool).scatter_(1, gi[:, :c["top"]], True)
    v = v.masked_fill(~kept.repeat_interleave(per, -1), -math.inf).sort(-1, descending=True).values[:, :c["k"] + 1]
    close |= (v[:, :-1] - v[:, 1:] < 1e-5).any(-1)
    best = torch.argmin(close.int())   # the first token that is decided
    return torch.where(close[:, None], logits[best], logits)


def _rows(experts, E):
    """(offsets, rows, slots) of the (token, choice) pairs in expert order; pairs without an expert come last."""
    key = experts.reshape(-1).long()
    key = torch.where(key < 0, E, key)
    rows = torch.sort(key, stable=True).indices
    offsets = torch.searchsorted(key[rows], torch.arange(E + 1, device=key.device)).int()
    slots = torch.empty_like(rows).scatter_(0, rows, torch.arange(rows.numel(), device=rows.device))
    slots = torch.where(key < E, slots, -1).int().view(experts.shape)
    return offsets, torch.where(key[rows] < E, rows, -1).int(), slots


def prepare(case, seed):
    c, gen = case, _gen(seed, 1)
    dtype = getattr(torch, c["dtype"])

    def normal(*shape, std=1.0, dtype=dtype):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0, std, generator=gen)

    if c["kind"] == "route":
        logits = _logits(c, gen).to(dtype)
        # balancing biases as a trainer moves them: a few hundred steps of 0.001 up or down
        bias = (torch.randn(c["E"], generator=gen, device="cuda") * 50).round() * 1e-3 if c["bias"] else None
        logits = _decided(c, logits, bias)
        logits[_none(c, gen)] = -math.inf
        s = {"case": c, "logits": logits, "bias": bias}
        if c["train"]:
            s["dweights"] = normal(c["T"], c["k"], dtype=torch.float32)
        return s
    if c["kind"] == "embed":
        # Zipf's law: the token of rank r is met in proportion to 1 / (r + 2.7)
        p = 1.0 / (torch.arange(c["V"], device="cuda", dtype=torch.float64) + 2.7)
        u = torch.rand(c["T"], generator=gen, device="cuda", dtype=torch.float64) * p.sum()
        rank = torch.searchsorted(p.cumsum(0), u).clamp_(max=c["V"] - 1)
        tokens = torch.randperm(c["V"], generator=gen, device="cuda")[rank]
        tokens[_none(c, gen)] = -1
        s = {"case": c, "tokens": tokens, "table": normal(c["V"], c["D"], std=0.02)}
        if c["train"]:
            s["dout"] = normal(c["T"], c["D"], std=1e-3)
        return s
    logits = _logits(c, gen)
    top = logits.sort(dim=-1, descending=True, stable=True)
    weights, experts = torch.softmax(top.values[:, :c["k"]], -1), top.indices[:, :c["k"]].int()
    none = _none(c, gen)
    experts[none], weights[none] = -1, 0.0
    offsets, rows, slots = _rows(experts, c["E"])
    s = {"case": c, "offsets": offsets, "rows": rows, "slots": slots, "weights": weights.contiguous(),
         "bounds": offsets.tolist(), "w": normal(c["E"], c["n"], c["m"], std=0.02)}
    R = c["T"] * c["k"]
    if c["kind"] == "up":
        s["x"] = normal(c["T"], c["n"])
        if c["dir"] == "bwd":
            s["dy"] = normal(R, c["m"], std=1e-3)
    else:
        s["x"] = normal(R, c["n"])
        if c["dir"] == "bwd":
            s["y"], s["dout"] = normal(R, c["m"]), normal(c["T"], c["m"], std=1e-3)
    return s


# ---- one pass ---------------------------------------------------------------------------------
def run(state):
    c = state["case"]
    if c["kind"] == "route":
        return _route_own(state) if own else _route_plain(state)
    if c["kind"] == "embed":
        return _embed_own(state) if own else _embed_plain(state)
    return _product_own(state) if own else _product_plain(state)


def _route_own(state):
    import paper_2607_19058_amd as P
    c = state["case"]
    how = dict(score=c["score"], renormalize=c["renorm"], scale=c["scale"])
    weights, experts = P.route(state["logits"], c["k"], bias=state["bias"], groups=c["groups"], top_groups=c["top"],
                               group_sum=2 if c["pair"] else 1, **how)
    plan = P.expert_rows(experts, c["E"])
    out = {"weights": weights, "experts": experts, "offsets": plan.offsets, "rows": plan.rows, "slots": plan.slots}
    if c["train"]:
        out["dlogits"] = P.route_backward(state["logits"], experts, state["dweights"], **how)
    return out


def _route_plain(state):
    c, E, k = state["case"], state["case"]["E"], state["case"]["k"]
    x = state["logits"].float()
    masked = x == -math.inf
    if c["score"] == "softmax":
        e = (x - x.amax(-1, keepdim=True).clamp(min=-3e38)).exp()
        s = e / e.sum(-1, keepdim=True).clamp(min=1e-38)
    else:
        s = 1.0 / (1.0 + (-x).exp())
    # without a bias the order of the scores is that of the logits, which no rounding changes
    v = x if state["bias"] is None else (s + state["bias"]).masked_fill(masked, -math.inf)
    if c["top"] < c["groups"]:
        by = v.view(-1, c["groups"], E // c["groups"]).sort(-1, descending=True).values[..., :2 if c["pair"] else 1]
        g = torch.where(by[..., 0] == -math.inf, -math.inf, by.masked_fill(by == -math.inf, 0.0).sum(-1))
        kept = g.sort(dim=-1, descending=True, stable=True).indices[:, :c["top"]]
        drop = torch.ones_like(g, dtype=torch.bool).scatter_(1, kept, False)
        v = v.masked_fill(drop.repeat_interleave(E // c["groups"], -1), -math.inf)
    best = v.sort(dim=-1, descending=True, stable=True)
    chosen, there = best.indices[:, :k], best.values[:, :k] != -math.inf
    sc = s.gather(1, chosen).masked_fill(~there, 0.0)
    total = sc.sum(-1, keepdim=True).clamp(min=1e-38) if c["renorm"] else 1.0
    experts = torch.where(there, chosen, -1).int()
    offsets, rows, slots = _rows(experts, E)
    out = {"weights": c["scale"] * (sc / total), "experts": experts, "offsets": offsets, "rows": rows, "slots": slots}
    if c["train"]:
        dw = state["dweights"].masked_fill(~there, 0.0) * c["scale"]
        ds = (dw - (dw * sc / total).sum(-1, keepdim=True)) / total if c["renorm"] else dw
        if c["score"] == "softmax":
            mean = 0.0 if c["renorm"] else (ds * sc).sum(-1, keepdim=True) * s
            dl = torch.zeros_like(x).scatter_(1, chosen, ds * sc) - mean
        else:
            dl = torch.zeros_like(x).scatter_(1, chosen, ds * sc * (1.0 - sc))
        out["dlogits"] = dl.to(state["logits"].dtype)
    return out


def _embed_own(state):
    import paper_2607_19058_amd as P
    c = state["case"]
    out = {"out": P.embed(state["tokens"], state["table"], scale=c["scale"])}
    if c["train"]:
        out["dtable"] = P.embed_grad(state["tokens"], state["dout"], c["V"], scale=c["scale"])
    return out


def _embed_plain(state):
    c, tokens, table = state["case"], state["tokens"], state["table"]
    there = tokens >= 0
    rows = table[tokens.clamp(min=0)].float().masked_fill(~there[:, None], 0.0)
    out = {"out": (rows * c["scale"]).to(table.dtype)}
    if c["train"]:
        d = torch.zeros(c["V"] + 1, c["D"], device="cuda")
        d.index_add_(0, torch.where(there, tokens, c["V"]), state["dout"].float())
        out["dtable"] = (d[:-1] * c["scale"]).to(table.dtype)
    return out


def _product_own(state):
    import paper_2607_19058_amd as P
    c, x, w = state["case"], state["x"], state["w"]
    plan = P.ExpertRows(state["offsets"], state["rows"], state["slots"])
    if c["kind"] == "up":
        if c["dir"] == "fwd":
            return {"y": P.expert_matmul(x, w, plan, gather=True)}
        dx = P.expert_matmul(state["dy"], w, plan, transpose=True, dtype=torch.float32)
        return {"dx": P.expert_combine(dx, plan, dtype=torch.bfloat16),
                "dw": P.expert_matmul_grad(x, state["dy"], plan, gather=True)}
    weights = state["weights"]
    if c["dir"] == "fwd":
        y = P.expert_matmul(x, w, plan, dtype=torch.float32)
        return {"out": P.expert_combine(y, plan, weights, dtype=torch.bfloat16)}
    dy, dweights = P.expert_combine_backward(state["dout"], state["y"], plan, weights)
    return {"dx": P.expert_matmul(state["dout"], w, plan, gather=True, transpose=True, scale=weights),
            "dw": P.expert_matmul_grad(x, dy, plan), "dweights": dweights}


def _experts(a, w, bounds):
    """Each expert's rows of `a` times its matrix; rows past the last expert's are zero. The experts hold different
    numbers of rows, so their products are one matrix product each."""
    y = torch.zeros(a.shape[0], w.shape[2], device="cuda")
    for e, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
        if hi > lo:
            torch.mm(a[lo:hi], w[e].float(), out=y[lo:hi])
    return y


def _outer(a, b, bounds, dtype):
    """Each expert's a^T b over its rows, rounded to `dtype`."""
    d = torch.zeros(len(bounds) - 1, a.shape[1], b.shape[1], dtype=dtype, device="cuda")
    for e, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
        if hi > lo:
            d[e] = torch.mm(a[lo:hi].T, b[lo:hi])
    return d


def _to_tokens(y, slots, weights):
    """Sum over a token's choices of its rows of y, times their weights."""
    picked = y[slots.long().clamp(min=0)] * (slots >= 0)[..., None]
    return (picked * weights[..., None] if weights is not None else picked).sum(1)


def _product_plain(state):
    c, w, bounds, slots = state["case"], state["w"], state["bounds"], state["slots"]
    there = (state["rows"] >= 0)[:, None]
    flat = state["rows"].long().clamp(min=0)
    token = flat // c["k"]
    x, weights = state["x"].float(), state["weights"]
    if c["kind"] == "up":
        if c["dir"] == "fwd":
            return {"y": _experts(x[token], w, bounds).bfloat16()}
        dy = state["dy"].float()
        dx = _experts(dy, w.transpose(1, 2), bounds)
        return {"dx": _to_tokens(dx, slots, None).bfloat16(), "dw": _outer(x[token], dy, bounds, w.dtype)}
    if c["dir"] == "fwd":
        return {"out": _to_tokens(_experts(x, w, bounds), slots, weights).bfloat16()}
    dout = state["dout"].float()
    dy = dout[token] * (weights.reshape(-1)[flat][:, None] * there)
    picked = state["y"][slots.long().clamp(min=0)].float() * (slots >= 0)[..., None]
    return {"dx": _experts(dy, w.transpose(1, 2), bounds).bfloat16(), "dw": _outer(x, dy, bounds, w.dtype),
            "dweights": (picked * dout[:, None]).sum(-1)}


# ---- work -------------------------------------------------------------------------------------
def work(case):
    c, T = case, case["T"]
    size = 4 if c["dtype"] == F32 else 2
    if c["kind"] == "route":
        E, R = c["E"], T * c["k"]
        # logits; weights, experts, rows and slots; in training the weights' gradients and the logits'
        nbytes = T * E * size + 16 * R + 4 * E + ((T * E * size + 4 * R) if c["train"] else 0)
        return {"bytes": nbytes, "flops": T * E * (8 if c["train"] else 4)}
    if c["kind"] == "embed":
        some = min(T, c["V"])   # rows of the table that are read, at most
        nbytes = (some + T) * c["D"] * size + 8 * T + ((T + c["V"]) * c["D"] * size if c["train"] else 0)
        return {"bytes": nbytes, "flops": T * c["D"] * (2 if c["train"] else 1)}
    E, R, n, m = c["E"], T * c["k"], c["n"], c["m"]
    # experts that have a row, for the shares that _logits draws (uniform on the simplex, R draws)
    active = E * R / (E - 1 + R)
    bwd = c["dir"] == "bwd"
    rows = (T * n + R * m) if c["kind"] == "up" else (R * n + T * m)
    nbytes = 2 * (active * n * m + rows)
    if bwd:   # the incoming rows as above, the outgoing ones, the weights' gradient of every expert
        nbytes += 2 * ((T if c["kind"] == "up" else R) * n + E * n * m)
        nbytes += 2 * R * m + 8 * R if c["kind"] == "down" else 0
    return {"bytes": int(nbytes), "flops": 2 * R * n * m * (2 if bwd else 1)}


# ---- the definition in 64 bits ----------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "route":
        return _route_exact(case, s)
    if case["kind"] == "embed":
        return _embed_exact(case, s)
    return _product_exact(case, s)


def _route_exact(c, s):
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    x, low = s["logits"].double(), -math.inf
    open_ = x > low
    if c["score"] == "softmax":
        z = torch.where(open_, x, -1e300)
        score = torch.where(open_, torch.exp(z - torch.logsumexp(z, -1, keepdim=True)), 0.0)
    else:
        score = torch.sigmoid(x)
    value = x.clone() if s["bias"] is None else torch.where(open_, score + s["bias"].double(), low)

    def first_best(v):   # the lowest index of the greatest value, and whether there is one
        top = v.max(-1, keepdim=True).values
        at = torch.where(v == top, torch.arange(v.shape[-1], device=v.device), v.shape[-1]).min(-1).values
        return at, top.squeeze(-1) > low

    if c["top"] < G:
        cells, worth = value.view(T, G, -1).clone(), torch.zeros(T, G, dtype=torch.float64, device="cuda")
        for i in range(2 if c["pair"] else 1):
            at, ok = first_best(cells)
            got = cells.gather(-1, at[..., None]).squeeze(-1)
            worth += torch.where(ok, got, 0.0 if i else low)
            cells.scatter_(-1, at[..., None], low)
        keep = torch.zeros(T, G, dtype=torch.bool, device="cuda")
        for _ in range(c["top"]):
            at, ok = first_best(worth)
            keep[torch.arange(T, device="cuda"), at] |= ok
            worth.scatter_(1, at[:, None], low)
        value = torch.where(keep[..., None].expand(T, G, E // G).reshape(T, E), value, low)
    experts = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    for j in range(k):
        at, ok = first_best(value)
        experts[:, j] = torch.where(ok, at, -1).int()
        value.scatter_(1, at[:, None], low)
    there = experts >= 0
    idx = experts.long().clamp(min=0)
    picked = torch.where(there, score.gather(1, idx), 0.0)
    S = picked.sum(1, keepdim=True)
    share = torch.where(S > 0, picked / S, 0.0)
    flat = torch.where(there, experts, E).reshape(-1).long()
    order = torch.argsort(flat * (T * k) + torch.arange(T * k, device="cuda"))
    count = torch.bincount(flat, minlength=E + 1)[:E]
    offsets = torch.cat([count.new_zeros(1), count.cumsum(0)])
    held = int(offsets[-1])
    rows = torch.where(torch.arange(T * k, device="cuda") < held, order, -1).int()
    slots = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
    slots[order[:held]] = torch.arange(held, device="cuda", dtype=torch.int32)
    out = {"weights": c["scale"] * (share if c["renorm"] else picked), "experts": experts, "offsets": offsets.int(),
           "rows": rows, "slots": slots.view(T, k)}
    if c["train"]:
        g = torch.where(there, s["dweights"].double(), 0.0) * c["scale"]
        if c["renorm"]:
            g = torch.where(there & (S > 0), (g - (g * share).sum(1, keepdim=True)) / S, 0.0)
        full = torch.zeros(T, E, dtype=torch.float64, device="cuda").scatter_add_(1, idx, g)
        if c["score"] == "softmax":
            out["dlogits"] = score * (full - (full * score).sum(1, keepdim=True))
        else:
            out["dlogits"] = full * score * (1 - score)
    return out


def _embed_exact(c, s):
    tokens = s["tokens"]
    keep = tokens >= 0
    out = torch.zeros(c["T"], c["D"], dtype=torch.float64, device="cuda")
    out[keep] = s["table"][tokens[keep]].double() * c["scale"]
    res = {"out": out}
    if c["train"]:
        d = torch.zeros(c["V"], c["D"], dtype=torch.float64, device="cuda")
        res["dtable"] = d.index_put_((tokens[keep],), s["dout"][keep].double() * c["scale"], accumulate=True)
    return res


def _product_exact(c, s):
    T, E, k, n, m = (c[i] for i in ("T", "E", "k", "n", "m"))
    slots, x = s["slots"].long(), s["x"]
    # whose row is at each place: from the slots, the inverse of the rows' order
    R = T * k
    pair = torch.zeros(R, dtype=torch.long, device="cuda")
    held = slots.reshape(-1) >= 0
    pair[slots.reshape(-1)[held]] = torch.arange(R, device="cuda")[held]
    up, bwd = c["kind"] == "up", c["dir"] == "bwd"
    f64 = dict(dtype=torch.float64, device="cuda")
    if not bwd:
        out = torch.zeros((R, m) if up else (T, m), **f64)
    else:
        dx, dw = torch.zeros((T, n) if up else (R, n), **f64), torch.zeros(E, n, m, **f64)
        dweights = torch.zeros(R, **f64)
    for e in range(E):
        lo, hi = s["bounds"][e], s["bounds"][e + 1]
        if lo == hi:
            continue
        mine = pair[lo:hi]
        token, weight = mine // k, s["weights"].reshape(-1)[mine].double()[:, None]
        a, mat = (x[token] if up else x[lo:hi]).double(), s["w"][e].double()
        if not bwd:
            y = a @ mat
            if up:
                out[lo:hi] = y
            else:
                out.index_add_(0, token, weight * y)
            continue
        d = s["dy"][lo:hi].double() if up else weight * s["dout"][token].double()
        back = d @ mat.T.contiguous()
        if up:
            dx.index_add_(0, token, back)
        else:
            dx[lo:hi] = back
            dweights[mine] = (s["y"][lo:hi].double() * s["dout"][token].double()).sum(1)
        dw[e] = a.T.contiguous() @ d
    if not bwd:
        return {"y" if up else "out": out}
    return {"dx": dx, "dw": dw} if up else {"dx": dx, "dw": dw, "dweights": dweights.view(T, k)}
