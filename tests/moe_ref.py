"""The mixture-of-experts operators from their definitions, in float64 on the CPU, and inputs for their tests."""
import math

import torch

U32 = 2.0**-24      # half an ulp of float32, relative
UBF = 2.0**-8       # of bf16 (8 significant bits: 1 and 1 + 2^-7 are neighbours)


def route(logits, k, score="softmax", bias=None, groups=1, top_groups=None, group_sum=1, renormalize=True, scale=1.0):
    """(weights, experts, scores, margin): margin is how far the choice is from another one (values in float64;
    equal values count as decided, by index)."""
    l = logits.double()
    T, E = l.shape
    top_groups = groups if top_groups is None else top_groups
    closed = l == -math.inf
    s = torch.zeros_like(l)
    for t in range(T):
        if score == "sigmoid":
            s[t] = 1 / (1 + torch.exp(-l[t]))
        elif not closed[t].all():
            z = torch.exp(l[t] - l[t].max())
            s[t] = z / z.sum()
    v = (l.clone() if bias is None else s + bias.double()).masked_fill(closed, -math.inf)
    v = torch.where(v.isnan(), math.inf, v)
    weights, experts = torch.zeros(T, k, dtype=torch.float64), torch.full((T, k), -1, dtype=torch.int32)
    margin = torch.full((T,), math.inf, dtype=torch.float64)

    def first(values, count, t):   # indices of the `count` highest, ties to the lowest index
        order = sorted(range(len(values)), key=lambda i: (-values[i], i))
        gaps = [values[a] - values[b] for a, b in zip(order[:count], order[1:]) if values[b] > -math.inf]
        gaps = [g for g in gaps if g > 0 and g == g]
        if gaps:
            margin[t] = min(float(margin[t]), min(gaps))
        return [i for i in order[:count] if values[i] > -math.inf]

    per = E // groups
    for t in range(T):
        val = v[t].tolist()
        if top_groups < groups:
            worth = []
            for g in range(groups):
                best = sorted((x for x in val[g * per:(g + 1) * per] if x > -math.inf), reverse=True)[:group_sum]
                worth.append(sum(best) if best else -math.inf)
            kept = first(worth, top_groups, t)
            val = [x if i // per in kept else -math.inf for i, x in enumerate(val)]
        for j, e in enumerate(first(val, k, t)):
            experts[t, j] = e
    w, there = s.gather(1, experts.long().clamp(min=0)), experts >= 0
    w = torch.where(there, w, 0.0)
    if renormalize:
        total = w.sum(1, keepdim=True)
        w = torch.where(total == 0, 0.0, w / total)
    return scale * w, experts, s, margin


def weights_of(logits, experts, score, renormalize, scale):
    """The weights as a differentiable function of float64 logits, for a given choice."""
    there = experts >= 0
    x = logits.gather(1, experts.long().clamp(min=0))
    if score == "softmax":
        mx = logits.max(1, keepdim=True).values.clamp(min=-1e30)
        w = torch.exp(x - mx) / torch.exp(logits - mx).sum(1, keepdim=True)
    else:
        w = 1 / (1 + torch.exp(-x))
    w = torch.where(there, w, 0.0)
    if renormalize:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / torch.where(total > 0, total, 1.0), 0.0)
    return scale * w


def logits_grad(logits, experts, dweights, score, renormalize, scale):
    l = logits.double()
    s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l.clamp(min=-1e30), 1).masked_fill(l == -math.inf, 0.0)
    there = experts >= 0
    at = experts.long().clamp(min=0)
    sc = torch.where(there, s.gather(1, at), 0.0)
    ds = torch.where(there, scale * dweights.double(), 0.0)
    if renormalize:
        S = sc.sum(1, keepdim=True)
        ds = torch.where(there & (S > 0), (ds - (ds * sc).sum(1, keepdim=True) / S) / S, 0.0)
    full = torch.zeros_like(l).scatter_add_(1, at, ds)
    if score == "sigmoid":
        return full * s * (1 - s)
    return s * (full - (full * s).sum(1, keepdim=True))


def rows(experts, E):
    flat = experts.reshape(-1).tolist()
    by = [[p for p, e in enumerate(flat) if e == i] for i in range(E)]
    order = [p for b in by for p in b]
    offsets = [0]
    for b in by:
        offsets.append(offsets[-1] + len(b))
    slots = torch.full((len(flat),), -1, dtype=torch.int32)
    slots[order] = torch.arange(len(order), dtype=torch.int32)
    return (torch.tensor(offsets, dtype=torch.int32),
            torch.tensor(order + [-1] * (len(flat) - len(order)), dtype=torch.int32), slots.view(experts.shape))


def matmul(x, w, offsets, row, k, gather=False, transpose=False, scale=None, absolute=False):
    """(T k, cols) in float64; `absolute`: of the absolute values (for error bounds)."""
    x, w = x.double(), w.double()
    if absolute:
        x, w = x.abs(), w.abs()
    R = row.numel()
    y = torch.zeros(R, w.shape[1] if transpose else w.shape[2], dtype=torch.float64)
    for e in range(w.shape[0]):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if hi > lo:
            a = x[row[lo:hi].long() // k] if gather else x[lo:hi]
            y[lo:hi] = a @ (w[e].T if transpose else w[e])
            if scale is not None:
                s = scale.double().reshape(-1)[row[lo:hi].long()]
                y[lo:hi] *= (s.abs() if absolute else s)[:, None]
    return y


def matmul_grad(x, dy, offsets, row, k, gather=False, absolute=False):
    x, dy = x.double(), dy.double()
    if absolute:
        x, dy = x.abs(), dy.abs()
    E = offsets.numel() - 1
    d = torch.zeros(E, x.shape[1], dy.shape[1], dtype=torch.float64)
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if hi > lo:
            a = x[row[lo:hi].long() // k] if gather else x[lo:hi]
            d[e] = a.T @ dy[lo:hi]
    return d


def draw_experts(T, E, k, gen, none=0.1, skew=True):
    """(T, k) distinct experts a token, some tokens without any and some with fewer; expert 0 popular, the last one unused."""
    score = torch.rand(T, E, generator=gen)
    if skew and E > 2:
        score[:, 0] += 0.5
        if k < E:
            score[:, E - 1] = -1.0
    experts = score.argsort(1, descending=True)[:, :k].int()
    experts[torch.rand(T, generator=gen) < none] = -1
    if k > 1:
        experts[torch.rand(T, generator=gen) < none, 1] = -1
    return experts
