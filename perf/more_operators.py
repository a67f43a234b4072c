"""Measured cases of a training step's loss and of what it keeps for the backward pass, in plain form and by the
package's operators.

A case names one of four passes:
  loss    softmax cross entropy of T tokens over a vocabulary of V, from rows x (T, d) and the head w, (d, V) or, with
          `tied`, the embedding's (V, d): loss and log-sum-exp of each token; with `train` also the gradients of x and w,
          from those of the losses (and, with `zloss`, of the log-sum-exps). A target outside [0, V) is no token
  keep    rows (R, C) to 8 bits and back: blocks of 32 values along a row share a power of two
  act     the activation between an expert's products, a = f(g) u, or f(g) without `gated`; with `train` g and u are kept
          in 8 bits, and the pass goes on with the backward one, which reads them: a once more, and the gradients of g, u
  grad    the experts' weights' gradient from rows that are kept in 8 bits: one a token (`gather`), or one a place
Fields besides: scale (of the logits), E experts, k experts a token, n x m the weight of one expert, pad (share of tokens
without a target or without experts), f (the activation), dtype.
"""
import math

import torch

own = False

F32, BF16 = "float32", "bfloat16"
LOSS = dict(kind="loss", d=2048, V=50304, tied=False, train=True, scale=1.0, zloss=False, pad=0.0, dtype=BF16)
KEEP = dict(kind="keep", dtype=BF16)
ACT = dict(kind="act", f="silu", gated=True, train=True, dtype=BF16)
GRAD = dict(kind="grad", k=2, gather=True, pad=0.0, dtype=BF16)
BLOCK = 32


def listed():
    def case(base, name, **kw):
        return dict(base, name=name, **kw)

    return [
        # one token scored while a model answers: the head's weights have to be read, nothing else counts
        case(LOSS, "loss_one_token", T=1, train=False),
        # the example's step: 2048 tokens of a small vocabulary, launches and latency
        case(LOSS, "loss_small_step", T=2048, d=128, V=512),
        # evaluation of a micro-batch of 1024 tokens with the benchmark model's head
        case(LOSS, "loss_micro_batch", T=1024, train=False),
        # a training step's 8192 tokens with the benchmark model's head: four products on the matrix cores
        case(LOSS, "loss_step", T=8192),
        # head and embedding share one table; the log-sum-exps are held near zero by a term of their own
        case(LOSS, "loss_tied", T=4096, tied=True, zloss=True),
        # widths that are no multiples of 8, padded tokens, scaled logits
        case(LOSS, "loss_odd", T=3001, d=1031, V=32003, scale=0.5, pad=0.05),
        # a few rows of the benchmark model's width: launches and latency
        case(KEEP, "keep_few_rows", R=16, C=2048),
        # the hidden rows of a step's 8192 tokens, two experts each: bound by memory
        case(KEEP, "keep_step", R=16384, C=8192),
        # gated experts over the same rows, forward and backward
        case(ACT, "act_step", R=16384, C=8192),
        # a float32 activation of odd width without a gate
        case(ACT, "act_odd", R=9003, C=2765, f="gelu_tanh", gated=False, dtype=F32),
        # the first product's weights' gradient of 32 experts with 512 uneven rows each, tokens' rows kept in 8 bits
        case(GRAD, "grad_step", T=8192, E=32, n=2048, m=8192),
        # odd widths, a kept row for each place, padded tokens
        case(GRAD, "grad_odd", T=3001, E=16, k=3, n=2765, m=1031, gather=False, pad=0.05),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):
        n = log(lo, hi)
        return n if rng.random() < 0.4 else max(lo, n // 64 * 64)

    kind = rng.choice(("loss", "loss", "loss", "keep", "act", "act", "grad"))
    while True:
        if kind == "loss":
            c = dict(LOSS, T=log(1, 8192), d=width(64, 4096), V=width(256, 60000), tied=rng.random() < 0.4,
                     train=rng.random() < 0.7, scale=rng.choice((1.0, 1.0, 0.5)), zloss=rng.random() < 0.3,
                     pad=rng.choice((0.0, 0.0, 0.05)))
        elif kind == "keep":
            c = dict(KEEP, R=log(1, 16384), C=width(32, 11008), dtype=rng.choice((F32, BF16, BF16)))
        elif kind == "act":
            c = dict(ACT, R=log(1, 16384), C=width(32, 11008), f=rng.choice(("silu", "silu", "gelu_tanh", "relu")),
                     gated=rng.random() < 0.6, train=rng.random() < 0.7, dtype=rng.choice((F32, BF16, BF16)))
        else:
            E = log(4, 64)
            c = dict(GRAD, T=log(1, 8192), E=E, k=min(E, rng.choice((1, 2, 2, 4))), n=width(64, 8192),
                     m=width(64, 8192), gather=rng.random() < 0.5, pad=rng.choice((0.0, 0.0, 0.05)))
            if E * c["n"] * c["m"] > 540_000_000:
                continue
        w = work(c)
        if w["flops"] <= {"loss": 5e12, "grad": 1e12}.get(kind, 1e18) and w["bytes"] <= 3e9:
            return c


# ---- inputs -----------------------------------------------------------------------------------
def _gen(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + k) & (2**62 - 1))
    return g


def _pack(x):
    """(codes int8, scales uint8) of rows x, padded with zeros to whole blocks: a block's scale is the smallest power of
    two from 2^-126 on of which its largest value is at most 127.5, kept with 127 added to its exponent."""
    R, C = x.shape
    blocks = torch.zeros(R, -(-C // BLOCK) * BLOCK, device=x.device)
    blocks[:, :C] = x
    blocks = blocks.view(R, -1, BLOCK)
    top = blocks.abs().amax(-1)
    m, e = torch.frexp(top)                               # top = m 2^e, m in [1/2, 1)
    e = torch.where(m > 127.5 / 128, e - 6, e - 7).clamp(min=-126)
    # (two factors, each of which float32 holds)
    codes = torch.round(torch.ldexp(torch.ldexp(blocks, -(e // 2)[..., None]), (e // 2 - e)[..., None]))
    return codes.clamp(-127, 127).to(torch.int8).view(R, -1), (e + 127).to(torch.uint8)


def _values(codes, scales, cols):
    """What the codes stand for, float32 (R, cols)."""
    s = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    return (codes.view(*scales.shape, BLOCK).float() * s[..., None]).view(codes.shape)[:, :cols]


def prepare(case, seed):
    c, gen = case, _gen(seed, 1)
    dtype = getattr(torch, c["dtype"])

    def normal(*shape, std=1.0, dtype=dtype):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0, std, generator=gen)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    if c["kind"] == "loss":
        T, d, V = c["T"], c["d"], c["V"]
        w = normal(V, d, std=0.02) if c["tied"] else normal(d, V, std=0.02)
        targets = (uniform(T) * V).long().clamp_(max=V - 1)
        # rows of a model that has learnt something: the target's logit is 0 to 14 above where chance would have it
        mine = (w[targets] if c["tied"] else w[:, targets].T).float()
        x = normal(T, d, dtype=torch.float32) + uniform(T, 1) * 14 / (c["scale"] * d * 0.02**2) * mine
        targets[uniform(T) < c["pad"]] = -1
        s = {"case": c, "x": x.to(dtype), "w": w, "targets": targets, "dlse": None}
        if c["train"]:   # a mean over the tokens, each with a weight near 1
            s["dloss"] = (0.5 + uniform(T)) / T
            if c["zloss"]:
                s["dlse"] = 2e-4 * (10 + uniform(T)) / T
        return s
    if c["kind"] == "keep":
        # rows with a few columns that are much larger than the others
        return {"case": c, "x": normal(c["R"], c["C"], dtype=torch.float32).mul_(
            0.2 + 0.5 * uniform(c["C"]) / uniform(c["C"]).clamp_(min=0.02)).to(dtype)}
    if c["kind"] == "act":
        s = {"case": c, "g": normal(c["R"], c["C"], std=1.5), "u": normal(c["R"], c["C"]) if c["gated"] else None}
        if c["train"]:
            s["da"] = normal(c["R"], c["C"], std=1e-3)
        return s
    T, E, k = c["T"], c["E"], c["k"]
    # experts differ in popularity; a token's are distinct; padded tokens have none
    share = uniform(E).clamp_(min=1e-3).log_().neg_().clamp_(min=1e-2).log_()
    score = share - uniform(T, E).clamp_(min=1e-9).log_().neg_().clamp_(min=1e-9).log_()
    experts = score.sort(dim=-1, descending=True, stable=True).indices[:, :k]
    experts[uniform(T) < c["pad"]] = E
    key = experts.reshape(-1)
    rows = torch.sort(key, stable=True).indices
    offsets = torch.searchsorted(key[rows], torch.arange(E + 1, device="cuda")).int()
    slots = torch.empty_like(rows).scatter_(0, rows, torch.arange(T * k, device="cuda"))
    codes, scales = _pack(normal(T if c["gather"] else T * k, c["n"]))
    return {"case": c, "codes": codes, "scales": scales, "dy": normal(T * k, c["m"], std=1e-3), "offsets": offsets,
            "rows": torch.where(key[rows] < E, rows, -1).int(), "slots": torch.where(key < E, slots, -1).int().view(T, k),
            "bounds": offsets.tolist()}


# ---- one pass ---------------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"loss": _loss_own, "keep": _keep_own, "act": _act_own, "grad": _grad_own}[kind](state)
    return {"loss": _loss_plain, "keep": _keep_plain, "act": _act_plain, "grad": _grad_plain}[kind](state)


def _loss_own(state):
    import paper_2607_19058_amd as P
    c, x, w, targets = state["case"], state["x"], state["w"], state["targets"]
    how = dict(tied=c["tied"], scale=c["scale"])
    loss, lse = P.head_loss(x, w, targets, **how)
    out = {"loss": loss, "lse": lse}
    if c["train"]:
        out["dx"], out["dw"] = P.head_loss_backward(x, w, targets, lse, state["dloss"], dlse=state["dlse"], **how)
    return out


def _loss_plain(state):
    c, x, w, targets = state["case"], state["x"].float(), state["w"].float(), state["targets"]
    if c["tied"]:
        w = w.T
    there, at = targets >= 0, targets.clamp(min=0)[:, None]
    z = (x @ w) * c["scale"]
    top = z.amax(-1, keepdim=True)
    lse = top.squeeze(-1) + (z - top).exp().sum(-1).log()
    out = {"loss": torch.where(there, lse - z.gather(1, at).squeeze(1), 0.0), "lse": torch.where(there, lse, 0.0)}
    if c["train"]:
        dloss = torch.where(there, state["dloss"], 0.0)[:, None]
        both = dloss if state["dlse"] is None else dloss + torch.where(there, state["dlse"], 0.0)[:, None]
        g = z.sub_(lse[:, None]).exp_().mul_(both)
        g.scatter_add_(1, at, -dloss)
        g *= c["scale"]
        dw = g.T @ x if c["tied"] else x.T @ g
        out["dx"], out["dw"] = (g @ w.T).bfloat16(), dw.bfloat16()
    return out


def _keep_own(state):
    import paper_2607_19058_amd as P
    return {"x": P.restore8(P.keep8(state["x"]), dtype=state["x"].dtype)}


def _keep_plain(state):
    x = state["x"]
    return {"x": _values(*_pack(x), x.shape[1]).to(x.dtype)}


def _act_own(state):
    import paper_2607_19058_amd as P
    c, g, u = state["case"], state["g"], state["u"]
    if not c["train"]:
        return {"a": P.expert_act(g, u, kind=c["f"])}
    a, kept = P.expert_act(g, u, kind=c["f"], keep=True)
    again, dg, du = P.expert_act_backward(state["da"], kept, kind=c["f"])
    return {"a": a, "again": again, "dg": dg, "du": du}


def _f_plain(g, f):
    """(f(g), f'(g))"""
    if f == "relu":
        return g.clamp(min=0.0), (g > 0).float()
    if f == "silu":
        s = 1.0 / (1.0 + (-g).exp())
        return g * s, s * (1.0 + g * (1.0 - s))
    # g / 2 (1 + tanh y) = g s(2 y)
    y2 = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g)
    s = 1.0 / (1.0 + (-y2).exp())
    return g * s, s + g * s * (1.0 - s) * 2 * math.sqrt(2 / math.pi) * (1.0 + 3 * 0.044715 * g * g)


def _act_plain(state):
    c, g, u = state["case"], state["g"], state["u"]
    dtype = g.dtype
    a = _f_plain(g.float(), c["f"])[0]
    out = {"a": (a if u is None else a * u.float()).to(dtype)}
    if c["train"]:
        da = state["da"].float()
        f, df = _f_plain(_values(*_pack(g), c["C"]), c["f"])
        uk = None if u is None else _values(*_pack(u), c["C"])
        out["again"] = (f if uk is None else f * uk).to(dtype)
        out["dg"] = (da * df if uk is None else da * uk * df).to(dtype)
        out["du"] = None if uk is None else (da * f).to(dtype)
    return out


def _grad_own(state):
    import paper_2607_19058_amd as P
    c = state["case"]
    plan = P.ExpertRows(state["offsets"], state["rows"], state["slots"])
    kept = P.Kept8(state["codes"], state["scales"], c["n"])
    return {"dw": P.expert_matmul_grad(kept, state["dy"], plan, gather=c["gather"])}


def _grad_plain(state):
    c, bounds = state["case"], state["bounds"]
    x, dy = _values(state["codes"], state["scales"], c["n"]), state["dy"].float()
    dw = torch.zeros(c["E"], c["n"], c["m"], dtype=torch.bfloat16, device="cuda")
    for e, (lo, hi) in enumerate(zip(bounds, bounds[1:])):   # one matrix product an expert, of its number of rows
        if hi > lo:
            a = x[state["rows"][lo:hi].long() // c["k"]] if c["gather"] else x[lo:hi]
            dw[e] = torch.mm(a.T, dy[lo:hi])
    return {"dw": dw}


# ---- work -------------------------------------------------------------------------------------
def work(case):
    c = case
    size = 4 if c["dtype"] == F32 else 2
    kept = 1 + 1 / BLOCK   # bytes of a value in 8 bits
    if c["kind"] == "loss":
        T, d, V = c["T"], c["d"], c["V"]
        # rows, the head and targets in, losses and log-sum-exps out; in training the two gradients, from two products more
        nbytes = 2 * (T * d + d * V) * (2 if c["train"] else 1) + 16 * T
        if c["train"]:
            nbytes += (8 if c["zloss"] else 4) * T
        return {"bytes": nbytes, "flops": 2 * T * d * V * (3 if c["train"] else 1)}
    if c["kind"] == "keep":   # to 8 bits, and back
        return {"bytes": int(c["R"] * c["C"] * 2 * (size + kept)), "flops": 4 * c["R"] * c["C"]}
    if c["kind"] == "act":
        n, ins = c["R"] * c["C"], 2 if c["gated"] else 1
        if not c["train"]:
            return {"bytes": n * size * (ins + 1), "flops": 8 * n}
        # g, u in, a and their 8 bits out; the gradient and these in, a and the gradients of g, u out
        return {"bytes": int(n * (size * (ins + 1) + size * (ins + 2) + 2 * kept * ins)), "flops": 24 * n}
    E, R, n, m = c["E"], c["T"] * c["k"], c["n"], c["m"]
    rows = c["T"] if c["gather"] else R
    return {"bytes": int(rows * n * kept + 2 * R * m + 2 * E * n * m), "flops": 2 * R * n * m}


# ---- the definition in 64 bits ----------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"loss": _loss_exact, "keep": _keep_exact, "act": _act_exact, "grad": _grad_exact}[case["kind"]](case, s)


def _loss_exact(c, s):
    T, a = c["T"], c["scale"]
    keep = torch.nonzero((s["targets"] >= 0) & (s["targets"] < c["V"])).squeeze(1)
    x, y = s["x"][keep].double(), s["targets"][keep]
    w = s["w"].double()
    by_word = w if c["tied"] else w.T.contiguous()
    logp = torch.log_softmax(a * (x @ by_word.T), dim=-1)
    n = torch.arange(keep.numel(), device="cuda")
    # log-sum-exp: a logit less its logarithm of a probability
    lse = a * (x * by_word[y]).sum(-1) - logp[n, y]

    def whole(v):
        return torch.zeros((T,) + v.shape[1:], dtype=torch.float64, device="cuda").index_copy_(0, keep, v)

    out = {"loss": whole(-logp[n, y]), "lse": whole(lse)}
    if c["train"]:
        d = s["dloss"][keep].double()
        both = d + s["dlse"][keep].double() if s["dlse"] is not None else d
        g = logp.exp() * (a * both)[:, None]
        g[n, y] -= a * d
        out["dx"] = whole(g @ by_word)
        dw = g.T.contiguous() @ x
        out["dw"] = dw if c["tied"] else dw.T
    return out


def _kept_exact(x):
    """x as 8 bits hold it: rounded to multiples of its block's power of two, which is found by trying the next."""
    R, C = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -C % BLOCK)).view(R, -1, BLOCK)
    top = v.abs().max(-1, keepdim=True).values
    step = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0**-126))) - 8).clamp(min=2.0**-126)
    for _ in range(4):
        step = torch.where(top > 127.5 * step, 2 * step, step)
    q = torch.round(v / step)
    return (torch.sign(q) * torch.minimum(q.abs(), torch.full_like(q, 127.0)) * step).view(R, -1)[:, :C]


def _keep_exact(c, s):
    return {"x": _kept_exact(s["x"])}


def _f_exact(g, f):
    if f == "relu":
        return torch.relu(g), torch.where(g > 0, 1.0, 0.0).double()
    if f == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g**3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 0.134145 * g * g)


def _act_exact(c, s):
    g, u = s["g"].double(), None if s["u"] is None else s["u"].double()
    f = _f_exact(g, c["f"])[0]
    out = {"a": f if u is None else f * u}
    if c["train"]:
        da = s["da"].double()
        f, df = _f_exact(_kept_exact(s["g"]), c["f"])
        uk = 1.0 if u is None else _kept_exact(s["u"])
        out["again"], out["dg"], out["du"] = f * uk, da * uk * df, None if u is None else da * f
    return out


def _grad_exact(c, s):
    R, n = s["codes"].shape[0], c["n"]
    step = torch.exp2(s["scales"].double() - 127).repeat_interleave(BLOCK, 1)
    x = (s["codes"].double() * step)[:, :n]
    # whose row is at each place: from the slots, the inverse of the rows' order
    T, k = s["slots"].shape
    flat = s["slots"].reshape(-1).long()
    token = torch.zeros(T * k, dtype=torch.long, device="cuda")
    pairs = torch.nonzero(flat >= 0).squeeze(1)
    token[flat[pairs]] = pairs // k
    dw = torch.zeros(c["E"], n, c["m"], dtype=torch.float64, device="cuda")
    for e in range(c["E"]):
        lo, hi = s["bounds"][e], s["bounds"][e + 1]
        if hi > lo:
            a = x[token[lo:hi]] if c["gather"] else x[lo:hi]
            dw[e] = a.T.contiguous() @ s["dy"][lo:hi].double()
    return {"dw": dw}
