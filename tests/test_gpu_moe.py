"""The mixture-of-experts operators on the GPU against their definitions in float64 (tests/moe_ref.py).

Tolerances, fixed from the arithmetic:
  weights     an exp of |x| < 32 is off by |x| half ulps of its argument and 2 of its own, sums of up to 1024 terms
              in a tree and two divisions by some 30 more: 64 half ulps of float32 (4e-6)
  products    a float32 sum of K products, in any order: K half ulps of the sum of absolute values (twice that, as
              the matrix instruction may truncate), and the final rounding (bf16: 2^-8 of the value)
  sums        as products with K terms
"""
import math

import pytest
import torch

import moe_ref as ref
import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator().manual_seed(seed)


def near(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = (got - want).abs() > bound
    assert not bad.any() and not got.isnan().any(), (what, int(bad.sum()), float((got - want).abs().max()))


def rounded(want, dtype):
    return want.abs() * (ref.UBF if dtype == BF else ref.U32) + 1e-38


# ---- routing ------------------------------------------------------------------------------------
ROUTES = [   # T, E, k, options
    (1, 1, 1, {}), (1, 128, 2, {}), (5, 8, 2, {}), (37, 16, 16, {}), (33, 17, 3, dict(score="sigmoid")), (64, 64, 4, {}),
    (50, 65, 2, dict(renormalize=False)), (129, 128, 8, dict(renormalize=False, scale=2.5)), (31, 129, 6, {}),
    (70, 256, 16, dict(score="sigmoid", renormalize=False)), (40, 257, 2, {}), (23, 512, 8, dict(renormalize=False)),
    (19, 700, 5, dict(score="sigmoid")), (9, 1024, 16, {}),
    (60, 32, 4, dict(bias=True)), (60, 128, 2, dict(bias=True, score="sigmoid", renormalize=False)),
    (60, 64, 6, dict(groups=8, top_groups=3)), (60, 60, 4, dict(groups=4, top_groups=2, bias=True, group_sum=2)),
    (60, 192, 6, dict(groups=6, top_groups=3, bias=True, group_sum=2, score="sigmoid", scale=1.5)),
    (60, 256, 8, dict(groups=64, top_groups=5, score="sigmoid")), (30, 640, 7, dict(groups=5, top_groups=2, bias=True)),
    (30, 512, 4, dict(groups=64, top_groups=1, bias=True, group_sum=2)), (40, 24, 3, dict(groups=24, top_groups=4)),
]


def _route_inputs(T, E, dtype, seed, bias):
    g = gen(seed)
    logits = torch.randn(T, E, generator=g) * 2
    logits = (logits * 8).round() / 8 if seed % 2 else logits   # a coarse grid: ties
    logits[torch.rand(T, E, generator=g) < 0.05] = -math.inf
    if T > 3:
        logits[1] = -math.inf                       # no open expert
        logits[2, :E - min(E, 2)] = -math.inf       # fewer open experts than choices
        logits[3] = 0.5                             # all alike
    b = (torch.randn(E, generator=g) * 50).round() * 1e-3 if bias else None
    return logits.to(dtype), b


@pytest.mark.parametrize("dtype", [F32, BF], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(ROUTES)), ids=lambda i: f"{ROUTES[i][0]}x{ROUTES[i][1]}-top{ROUTES[i][2]}-{i}")
def test_route_and_backward(case, dtype):
    T, E, k, opt = ROUTES[case]
    opt = dict(opt)
    logits, bias = _route_inputs(T, E, dtype, case, opt.pop("bias", False))
    how = {n: opt[n] for n in ("score", "renormalize", "scale") if n in opt}
    wide = torch.full((T, E + 3), 9.0, dtype=dtype)   # rows with a stride: nothing past E is read
    wide[:, :E] = logits
    want_w, want_e, _, margin = ref.route(logits, k, bias=bias, **opt)
    sure = margin > 1e-5 if bias is not None else margin > 0
    assert sure.float().mean() > 0.8
    for src in (logits.to(DEV), wide.to(DEV)[:, :E]):
        w, e = P.route(src, k, bias=None if bias is None else bias.to(DEV), **opt)
        assert torch.equal(e.cpu()[sure], want_e[sure])
        near(w[sure.to(DEV)], want_w[sure], 64 * ref.U32 * want_w[sure].abs() + 1e-30, "weights")
        # the gradient, for the choice that was made
        e = e.cpu()
        dw = torch.randn(T, k, generator=gen(case + 100))
        args = dict(dict(score="softmax", renormalize=True, scale=1.0), **how)
        want = ref.logits_grad(logits, e, dw, **args)
        size = ref.logits_grad(logits, e, dw.abs(), args["score"], False, abs(args["scale"])).abs().max(1, keepdim=True).values
        size = torch.maximum(size, dw.abs().max(1, keepdim=True).values.double() * abs(args["scale"]))
        got = P.route_backward(src, e.to(DEV), dw.to(DEV), **how)
        assert got.dtype == dtype and got.is_contiguous()
        near(got, want, 64 * ref.U32 * size + rounded(want, dtype), "dlogits")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_backward_against_differences(score, renormalize):
    """Central differences of the float64 weights: error O(h^2) = 1e-8 of values of order 1, and their rounding 1e-11."""
    T, E, k, h = 6, 24, 3, 1e-4
    logits = torch.randn(T, E, generator=gen(5))
    w, e = P.route(logits.to(DEV), k, score=score, renormalize=renormalize, scale=1.5)
    dw = torch.randn(T, k, generator=gen(6))
    got = P.route_backward(logits.to(DEV), e, dw.to(DEV), score=score, renormalize=renormalize, scale=1.5).cpu().double()

    def f(l):
        return (ref.weights_of(l, e.cpu(), score, renormalize, 1.5) * dw.double()).sum(1)

    for j in range(E):
        d = torch.zeros(T, E, dtype=torch.float64)
        d[:, j] = h
        want = (f(logits.double() + d) - f(logits.double() - d)) / (2 * h)
        assert (got[:, j] - want).abs().max() < 1e-5


def test_route_of_special_values():
    inf, nan = math.inf, math.nan
    l = torch.tensor([[0.0, nan, 1.0, 2.0], [0.0, inf, 1.0, 2.0], [-inf, -3e38, 3e38, 0.0], [88.0, 89.0, -100.0, 90.0],
                      [-inf, -inf, -inf, 5.0]])
    w, e = P.route(l.to(DEV), 2)
    assert e.cpu().tolist() == [[1, 3], [1, 3], [2, 3], [3, 1], [3, -1]]
    w = w.cpu()
    assert w[:2].isnan().all()                       # shown, not hidden
    assert w[2].tolist() == [1.0, 0.0] and w[4].tolist() == [1.0, 0.0]
    assert torch.allclose(w[3].double(), torch.softmax(torch.tensor([90.0, 89.0], dtype=torch.float64), 0), rtol=1e-6)
    # the lowest finite value of the type is no mask: such an expert is open, with a score of zero
    low = torch.full((2, 6), torch.finfo(BF).min, dtype=BF)
    low[1, 4] = 1.0
    w, e = P.route(low.to(DEV), 3, renormalize=False)
    assert e.cpu().tolist() == [[0, 1, 2], [4, 0, 1]]
    assert torch.allclose(w.cpu(), torch.tensor([[1 / 6] * 3, [1.0, 0.0, 0.0]]))
    d = P.route_backward(l[4:].to(DEV), torch.tensor([[3, -1]], dtype=torch.int32, device=DEV), torch.ones(1, 2, device=DEV))
    assert d.cpu().tolist() == [[0.0] * 4]


def test_route_of_no_tokens():
    w, e = P.route(torch.empty(0, 8, device=DEV), 2)
    assert w.shape == (0, 2) and e.shape == (0, 2)
    assert P.route_backward(torch.empty(0, 8, device=DEV), e, w).shape == (0, 8)
    plan = P.expert_rows(e, 8)
    assert plan.offsets.cpu().tolist() == [0] * 9 and plan.rows.numel() == 0 and plan.slots.shape == (0, 2)


# ---- order --------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 2, 128), (63, 1, 8), (500, 3, 65), (8192, 2, 128), (4096, 4, 511),
                                   (16385, 1, 8), (9000, 3, 512), (20011, 2, 1024), (70001, 1, 1)])
def test_expert_rows(T, k, E):
    experts = torch.randint(-1, E + (E < 1024), (T, k), generator=gen(T), dtype=torch.int32)
    if T == 20011:
        experts[: T // 2] = 7   # a run of one expert over several work-groups
    plan = P.expert_rows(experts.to(DEV), E)
    key = torch.where((experts < 0) | (experts >= E), E, experts).reshape(-1)
    order = torch.argsort(key, stable=True).int()
    held = int((key < E).sum())
    assert torch.equal(plan.offsets.cpu(), torch.searchsorted(key[order.long()].contiguous(), torch.arange(E + 1)).int())
    assert torch.equal(plan.rows.cpu()[:held], order[:held]) and (plan.rows.cpu()[held:] == -1).all()
    slots = torch.full((T * k,), -1, dtype=torch.int32)
    slots[order[:held].long()] = torch.arange(held, dtype=torch.int32)
    assert torch.equal(plan.slots.cpu().reshape(-1), slots)


# ---- products -----------------------------------------------------------------------------------
SHAPES = [   # T, E, k, n, m
    (1, 4, 2, 64, 64), (1, 1, 1, 1, 1), (3, 2, 1, 8, 16), (7, 5, 2, 33, 17), (40, 3, 2, 128, 200), (64, 8, 2, 256, 320),
    (130, 4, 3, 72, 136), (257, 2, 1, 65, 129), (300, 6, 2, 320, 96), (97, 9, 4, 31, 250), (600, 3, 2, 264, 392),
    (16, 64, 2, 128, 512), (1000, 2, 1, 520, 264),
]


def _products(i, none=0.1):
    T, E, k, n, m = SHAPES[i]
    g = gen(i)
    experts = ref.draw_experts(T, E, k, g, none)
    plan = P.expert_rows(experts.to(DEV), E)
    return T, E, k, n, m, g, plan, ref.rows(experts, E)


def _matmul_bound(x, w, off, row, k, K, dtype, want, **kw):
    return 2 * (K + 8) * ref.U32 * ref.matmul(x, w, off, row, k, absolute=True, **kw) + rounded(want, dtype)


@pytest.mark.parametrize("i", range(len(SHAPES)), ids=lambda i: "x".join(map(str, SHAPES[i])))
@pytest.mark.parametrize("transpose", [False, True], ids=["forward", "backward"])
def test_expert_matmul(i, transpose):
    T, E, k, n, m, g, plan, (off, row, _) = _products(i)
    K, cols = (m, n) if transpose else (n, m)
    w = torch.randn(E, n, m, generator=g).to(BF)
    scale = torch.randn(T, k, generator=g)
    for gather in (False, True):
        x = torch.randn(T if gather else T * k, K, generator=g).to(BF)
        for dtype, s in ((BF, None), (F32, scale)):
            kw = dict(gather=gather, transpose=transpose, scale=s)
            want = ref.matmul(x, w, off, row, k, **kw)
            got = P.expert_matmul(x.to(DEV), w.to(DEV), plan, gather=gather, transpose=transpose,
                                  scale=None if s is None else s.to(DEV), dtype=dtype)
            assert got.dtype == dtype
            near(got, want, _matmul_bound(x, w, off, row, k, K, dtype, want, **kw), (gather, dtype))
            again = P.expert_matmul(x.to(DEV), w.to(DEV), plan, gather=gather, transpose=transpose,
                                    scale=None if s is None else s.to(DEV), dtype=dtype)
            assert torch.equal(got, again)


@pytest.mark.parametrize("i", range(len(SHAPES)), ids=lambda i: "x".join(map(str, SHAPES[i])))
def test_expert_matmul_grad(i):
    T, E, k, n, m, g, plan, (off, row, _) = _products(i)
    dy = torch.randn(T * k, m, generator=g).to(BF)
    K = int((off[1:] - off[:-1]).max())
    for gather in (False, True):
        x = torch.randn(T if gather else T * k, n, generator=g).to(BF)
        want = ref.matmul_grad(x, dy, off, row, k, gather)
        got = P.expert_matmul_grad(x.to(DEV), dy.to(DEV), plan, gather=gather)
        bound = 2 * (K + 8) * ref.U32 * ref.matmul_grad(x, dy, off, row, k, gather, absolute=True) + rounded(want, BF)
        near(got, want, bound, gather)


@pytest.mark.parametrize("shift", [0, 1, 4], ids=["aligned", "odd", "8-byte"])
def test_products_of_strided_views(shift):
    """Row strides above the row, slices that leave a gap, first elements at any position; what surrounds the output
    stays as it was, and what surrounds the inputs (NaN) is not used."""
    T, E, k, n, m = 50, 3, 2, 72, 88
    g = gen(11)
    experts = ref.draw_experts(T, E, k, g)
    off, row, _ = ref.rows(experts, E)
    plan = P.expert_rows(experts.to(DEV), E)

    def view(*shape):   # a view inside a larger buffer of NaN
        big = torch.full([s + 3 for s in shape[:-1]] + [shape[-1] + 16], math.nan, dtype=BF)
        v = big[tuple(slice(0, s) for s in shape[:-1]) + (slice(shift, shift + shape[-1]),)]
        v.copy_(torch.randn(shape, generator=g))
        return v.contiguous(), big.to(DEV)[tuple(slice(0, s) for s in shape[:-1]) + (slice(shift, shift + shape[-1]),)]

    x, xd = view(T, n)
    w, wd = view(E, n, m)
    dy, dyd = view(T * k, m)
    want = ref.matmul(x, w, off, row, k, gather=True)
    near(P.expert_matmul(xd, wd, plan, gather=True), want, _matmul_bound(x, w, off, row, k, n, BF, want, gather=True), "forward")
    want = ref.matmul(dy, w, off, row, k, transpose=True)
    near(P.expert_matmul(dyd, wd, plan, transpose=True), want,
         _matmul_bound(dy, w, off, row, k, m, BF, want, transpose=True), "backward")
    big = torch.full((E + 1, n + 3, m + 16), 7.0, dtype=BF, device=DEV)
    out = big[:E, :n, shift:shift + m]
    assert P.expert_matmul_grad(xd, dyd, plan, gather=True, out=out) is out
    want = ref.matmul_grad(x, dy, off, row, k, True)
    near(out, want, 2 * (T * k) * ref.U32 * ref.matmul_grad(x, dy, off, row, k, True, absolute=True) + rounded(want, BF), "grad")
    out.fill_(7.0)
    assert (big == 7.0).all()


def test_products_keep_nonfinite_values_in_their_rows():
    """An infinity or NaN in one row of x shows in that row of y alone, also with lengths that end inside a tile."""
    T, E, n, m = 20, 2, 36, 50
    experts = (torch.arange(T) % 2).int()[:, None]
    plan = P.expert_rows(experts.to(DEV), E)
    g = gen(3)
    x, w = torch.randn(T, n, generator=g).to(BF), torch.randn(E, n, m, generator=g).to(BF)
    x[4, 35], x[9, 0] = math.inf, math.nan
    y = P.expert_matmul(x.to(DEV), w.to(DEV), plan, gather=True).cpu()
    place = plan.slots.cpu()[:, 0].tolist()
    for t in range(T):
        if t in (4, 9):
            assert not y[place[t]].isfinite().any()
        else:
            assert y[place[t]].isfinite().all()
    w[1, 35, 7] = math.nan
    x = torch.randn(T, n, generator=g).to(BF)
    y = P.expert_matmul(x.to(DEV), w.to(DEV), plan, gather=True).cpu()
    assert y[10:, 7].isnan().all() and y[:10].isfinite().all() and y.isnan().sum() == 10


def test_products_without_any_expert():
    """Every token without experts: rows, sums and gradients are all zero (and overwritten)."""
    T, E, k, n, m = 70, 3, 2, 40, 48
    experts = torch.full((T, k), -1, dtype=torch.int32, device=DEV)
    plan = P.expert_rows(experts, E)
    x, w = torch.randn(T, n, device=DEV).to(BF), torch.randn(E, n, m, device=DEV).to(BF)
    dy = torch.randn(T * k, m, device=DEV).to(BF)
    out = torch.full((E, n, m), math.nan, dtype=BF, device=DEV)
    assert not P.expert_matmul(x, w, plan, gather=True).any()
    assert not P.expert_matmul(dy, w, plan, transpose=True).any()
    assert not P.expert_matmul_grad(x, dy, plan, gather=True, out=out).any()
    assert not P.expert_combine(dy, plan, torch.ones(T, k, device=DEV)).any()
    d, dw = P.expert_combine_backward(torch.randn(T, m, device=DEV).to(BF), dy, plan)
    assert not d.any() and not dw.any()


def test_products_of_no_tokens():
    plan = P.expert_rows(torch.empty(0, 2, dtype=torch.int32, device=DEV), 3)
    x, w, dy = (torch.empty(s, dtype=BF, device=DEV) for s in ((0, 8), (3, 8, 16), (0, 16)))
    assert P.expert_matmul(x, w, plan, gather=True).shape == (0, 16)
    assert not P.expert_matmul_grad(x, dy, plan, out=torch.ones(3, 8, 16, dtype=BF, device=DEV)).any()
    assert P.expert_combine(dy, plan).shape == (0, 16)
    d, dw = P.expert_combine_backward(dy, dy, plan)
    assert d.shape == (0, 16) and dw.shape == (0, 2)


# ---- weighted sums of expert rows -----------------------------------------------------------------
@pytest.mark.parametrize("ydtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,E,k,m", [(1, 4, 2, 8), (33, 8, 2, 256), (50, 5, 4, 67), (40, 3, 1, 2048), (9, 20, 16, 4100), (5, 2, 2, 1)])
def test_combine_and_backward(T, E, k, m, ydtype):
    g = gen(T)
    experts = ref.draw_experts(T, E, k, g)
    plan = P.expert_rows(experts.to(DEV), E)
    off, row, slots = ref.rows(experts, E)
    y, weights = torch.randn(T * k, m, generator=g).to(ydtype), torch.randn(T, k, generator=g)
    dout = torch.randn(T, m, generator=g).to(BF)
    there = (slots >= 0)[..., None]
    picked = y.double()[slots.long().clamp(min=0)] * there
    for w in (weights, None):
        wd = torch.ones(T, k).double() if w is None else w.double()
        terms = picked * wd[..., None]
        for dtype in (BF, F32):
            got = P.expert_combine(y.to(DEV), plan, None if w is None else w.to(DEV), dtype=dtype)
            near(got, terms.sum(1), (k + 1) * ref.U32 * terms.abs().sum(1) + rounded(terms.sum(1), dtype), dtype)
        dy, dw = P.expert_combine_backward(dout.to(DEV), y.to(DEV), plan, None if w is None else w.to(DEV))
        want = torch.zeros(T * k, m, dtype=torch.float64)
        held = int(off[-1])
        pair = row[:held].long()
        want[:held] = dout.double()[pair // k] * wd.reshape(-1)[pair][:, None]
        near(dy, want, ref.U32 * want.abs() + rounded(want, BF), "dy")
        products = picked * dout.double()[:, None]
        near(dw, products.sum(-1), (m + 2) * ref.U32 * products.abs().sum(-1) + 1e-38, "dweights")
    assert P.expert_combine(y.to(DEV), plan).dtype == ydtype


# ---- embedding ----------------------------------------------------------------------------------
EMBEDS = [   # T, V, D, dtype, ids
    (1, 1, 1, F32, torch.int64), (16, 50304, 256, BF, torch.int64), (300, 40, 67, BF, torch.int32), (1000, 3, 129, F32, torch.int64),
    (65, 7, 2056, BF, torch.int64), (5000, 2000, 40, BF, torch.int32), (16385, 900, 33, F32, torch.int64),
    (20000, 300000, 16, BF, torch.int64), (129, 1 << 20, 8, F32, torch.int32), (4096, 1, 24, BF, torch.int64),
]


@pytest.mark.parametrize("T,V,D,dtype,idt", EMBEDS, ids=lambda v: str(v).replace("torch.", ""))
def test_embed_and_grad(T, V, D, dtype, idt):
    g = gen(T + V)
    tokens = (torch.rand(T, generator=g) ** 4 * V).long().clamp(max=V - 1)   # frequent low ids, long runs of them
    tokens[torch.rand(T, generator=g) < 0.1] = -1
    tokens[torch.rand(T, generator=g) < 0.02] = V          # beyond the table: no token either
    tokens = tokens.to(idt)
    there = (tokens >= 0) & (tokens < V)
    table = torch.randn(V, D, generator=g).to(dtype)
    scale = 0.375
    want = torch.where(there[:, None], table[tokens.long().clamp(0, V - 1)].double() * scale, 0.0)
    near(P.embed(tokens.to(DEV), table.to(DEV), scale=scale), want, ref.U32 * want.abs() + rounded(want, dtype), "embed")
    dout = torch.randn(T, D, generator=g).to(dtype)
    kept = tokens[there].long()
    want = torch.zeros(V, D, dtype=torch.float64).index_add_(0, kept, dout[there].double() * scale)
    size = torch.zeros(V, D, dtype=torch.float64).index_add_(0, kept, dout[there].double().abs() * scale)
    count = torch.bincount(kept, minlength=V)[:, None]
    got = P.embed_grad(tokens.to(DEV), dout.to(DEV), V, scale=scale)
    near(got, want, (count + 2) * ref.U32 * size + rounded(want, dtype), "dtable")
    assert torch.equal(got, P.embed_grad(tokens.to(DEV), dout.to(DEV), V, scale=scale))
    assert not got[(count[:, 0] == 0).to(DEV)].any()


def test_embed_of_strided_tables_and_no_tokens():
    V, D, T = 50, 70, 90
    g = gen(2)
    big = torch.randn(V, D + 9, generator=g)
    tokens = torch.randint(0, V, (T,), generator=g)
    table = big.to(DEV)[:, 3:3 + D]
    assert torch.equal(P.embed(tokens.to(DEV), table).cpu(), big[:, 3:3 + D][tokens])
    dout = torch.randn(T, D + 5, generator=g).to(DEV)[:, 2:2 + D]
    room = torch.full((V, D + 9), 7.0, device=DEV)
    out = room[:, 3:3 + D]
    assert P.embed_grad(tokens.to(DEV), dout, V, out=out) is out
    want = torch.zeros(V, D, dtype=torch.float64).index_add_(0, tokens, dout.cpu().double())
    near(out, want, 1e-5 + 0 * want, "dtable")
    out.fill_(7.0)
    assert (room == 7.0).all()
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    assert P.embed(none, table).shape == (0, D)
    for v in (V, 300001):   # both sorts
        assert not P.embed_grad(none, dout[:0], v, out=torch.full((v, D), math.nan, device=DEV)).any()


def test_embed_grad_against_differences():
    """The lookup is linear in the table: a difference of 1 in one entry moves <dout, out> by that entry's gradient."""
    V, D, T = 6, 5, 40
    g = gen(9)
    tokens, table, dout = torch.randint(0, V, (T,), generator=g), torch.zeros(V, D), torch.randn(T, D, generator=g)
    got = P.embed_grad(tokens.to(DEV), dout.to(DEV), V, scale=2.0).cpu()
    for v in range(V):
        for c in range(D):
            table[v, c] = 1.0
            out = P.embed(tokens.to(DEV), table.to(DEV), scale=2.0).cpu()
            assert abs(float((out.double() * dout.double()).sum()) - float(got[v, c])) < 1e-4
            table[v, c] = 0.0


# ---- how they are called --------------------------------------------------------------------------
def _layer(logits, x, w1, w2, dout, stream=None):
    weights, experts = P.route(logits, 2, stream=stream)
    plan = P.expert_rows(experts, w1.shape[0], stream=stream)
    h = P.expert_matmul(x, w1, plan, gather=True, stream=stream)
    y = P.expert_matmul(h, w2, plan, dtype=F32, stream=stream)
    out = P.expert_combine(y, plan, weights, dtype=BF, stream=stream)
    dy, dweights = P.expert_combine_backward(dout, y, plan, weights, stream=stream)
    dh = P.expert_matmul(dout, w2, plan, gather=True, transpose=True, scale=weights, stream=stream)
    dw2 = P.expert_matmul_grad(h, dy, plan, stream=stream)
    dx = P.expert_combine(P.expert_matmul(dh, w1, plan, transpose=True, dtype=F32, stream=stream), plan, dtype=BF, stream=stream)
    dw1 = P.expert_matmul_grad(x, dh, plan, gather=True, stream=stream)
    return out, dx, dw1, dw2, P.route_backward(logits, experts, dweights, stream=stream)


def _layer_inputs(T=100, E=8, d=64, f=128, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def r(*s, dtype=BF):
        return torch.randn(s, generator=g, device=DEV).to(dtype)
    return r(T, E, dtype=F32), r(T, d), r(E, d, f), r(E, f, d), r(T, d)


def test_layer_gradient_against_differences():
    """The whole layer's gradients of logits, input and weights against central differences of a float64 layer with
    the same choices: bf16 roundings of h, dy and dh (2^-8 each) leave some 2 per cent of a directional derivative."""
    logits, x, w1, w2, dout = _layer_inputs(T=24, E=4, d=16, f=32)
    _, dx, dw1, dw2, dlogits = _layer(logits, x, w1, w2, dout)
    _, experts = P.route(logits, 2)
    e = experts.cpu().long()
    l, xx, a, b, dd = (t.cpu().double() for t in (logits, x, w1, w2, dout))

    def loss(l, xx, a, b):
        p = torch.softmax(l, 1).gather(1, e)
        p = p / p.sum(1, keepdim=True)
        y = torch.einsum("td,tkdf->tkf", xx, a[e])
        y = torch.einsum("tkf,tkfd->tkd", y, b[e])
        return float(((y * p[..., None]).sum(1) * dd).sum())

    for which, grad in ((0, dlogits), (1, dx), (2, dw1), (3, dw2)):
        args = [l, xx, a, b]
        direction = grad.cpu().double()
        h = 1e-4 / float(direction.abs().max())
        up, down = list(args), list(args)
        up[which], down[which] = args[which] + h * direction, args[which] - h * direction
        slope = (loss(*up) - loss(*down)) / (2 * h)
        assert abs(slope / float(direction.square().sum()) - 1) < 0.02, which


def test_layer_on_another_stream():
    inputs = _layer_inputs()
    want = _layer(*inputs)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = _layer(*inputs, stream=s)
    handle = _layer(*inputs, stream=s.cuda_stream)
    s.synchronize()
    for a, b, c in zip(want, got, handle):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_layer_in_a_graph():
    """Captured once, replayed on new inputs with eager work between the replays: the same bits as the eager calls."""
    inputs = _layer_inputs()
    tokens = torch.randint(0, 300, (2000,), device=DEV)
    dout = torch.randn(2000, 40, device=DEV)

    def everything():
        return (*_layer(*inputs), P.embed_grad(tokens, dout, 300), P.embed_grad(tokens, dout, 300000))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        everything()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = everything()
    for seed in range(2, 6):
        for t, new in zip(inputs, _layer_inputs(seed=seed)):
            t.copy_(new)
        tokens.random_(0, 300, generator=torch.Generator(device=DEV).manual_seed(seed))
        want = everything()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


def test_refusals_of_the_binding():
    logits, x, w1, w2, dout = _layer_inputs()
    weights, experts = P.route(logits, 2)
    plan = P.expert_rows(experts, 8)
    h = torch.zeros(200, 128, dtype=BF, device=DEV)
    for err, call in (
            (ValueError, lambda: P.route(logits, 0)), (ValueError, lambda: P.route(logits, 9)),
            (ValueError, lambda: P.route(logits, 2, score="tanh")), (ValueError, lambda: P.route(logits, 2, groups=3)),
            (ValueError, lambda: P.route(logits, 3, groups=4, top_groups=1)), (ValueError, lambda: P.route(logits, 2, group_sum=2)),
            (ValueError, lambda: P.route(logits, 2, bias=torch.zeros(7, device=DEV))),
            (TypeError, lambda: P.route(logits, 2, bias=torch.zeros(8, device=DEV, dtype=BF))),
            (ValueError, lambda: P.route(logits.T, 2)), (ValueError, lambda: P.route(logits, 2, scale=math.nan)),
            (TypeError, lambda: P.route(logits.double(), 2)), (ValueError, lambda: P.route(logits[0], 2)),
            (ValueError, lambda: P.route(logits[:1].expand(100, 8), 2)),
            (ValueError, lambda: P.route_backward(logits, experts[:50], weights)),
            (TypeError, lambda: P.route_backward(logits, experts.long(), weights)),
            (ValueError, lambda: P.expert_rows(experts, 0)), (ValueError, lambda: P.expert_rows(experts, 1025)),
            (ValueError, lambda: P.expert_rows(experts.T, 8)), (TypeError, lambda: P.expert_rows(experts.long(), 8)),
            (ValueError, lambda: P.expert_matmul(x, w1, plan)), (ValueError, lambda: P.expert_matmul(h, w1, plan)),
            (ValueError, lambda: P.expert_matmul(x, w1[:7], plan, gather=True)),
            (TypeError, lambda: P.expert_matmul(x.float(), w1, plan, gather=True)),
            (TypeError, lambda: P.expert_matmul(x, w1, plan, gather=True, dtype=torch.float16)),
            (ValueError, lambda: P.expert_matmul(x, w1, plan, gather=True, scale=weights[:50])),
            (ValueError, lambda: P.expert_matmul(x, w1.transpose(1, 2), plan, gather=True)),
            (ValueError, lambda: P.expert_matmul(x, w1[:1].expand(8, 64, 128), plan, gather=True)),
            (ValueError, lambda: P.expert_matmul_grad(x, h[:100], plan, gather=True)),
            (ValueError, lambda: P.expert_matmul_grad(x, h, plan, gather=True, out=w2)),
            (ValueError, lambda: P.expert_combine(x, plan)), (ValueError, lambda: P.expert_combine(h, plan, weights[:50])),
            (ValueError, lambda: P.expert_combine_backward(dout, h, plan)),
            (ValueError, lambda: P.embed(experts, x)), (TypeError, lambda: P.embed(weights[:, 0], x)),
            (ValueError, lambda: P.embed(experts[:, 0], x)), (TypeError, lambda: P.embed(experts[:, 0].contiguous(), x.half())),
            (ValueError, lambda: P.embed_grad(experts[:50, 0].contiguous(), dout, 8)),
            (ValueError, lambda: P.embed_grad(experts[:, 0].contiguous(), dout, 0)),
            (ValueError, lambda: P.embed_grad(experts[:, 0].contiguous(), dout, 8, out=x)),
            (TypeError, lambda: P.embed(experts[:, 0].contiguous().cpu(), x))):
        with pytest.raises(err):
            call()
