"""Rows kept in 8 bits, the experts' activation and the weights' gradient from kept rows on the GPU, against their definitions
in float64 (tests/kept_ref.py, tests/moe_ref.py).

Tolerances, fixed from the arithmetic:
  codes, scales, restored values   none: powers of two and one rounding to a whole number, which float32 does exactly
  activations                      kept_ref.act_bound, a product or two with u and da (2 half ulps of float32 each), and the
                                   final rounding (bf16: 2^-8 of the value)
  weights' gradient                as of rows in bf16: 4 K + 16 half ulps of the sum of absolute values, and the rounding;
                                   2^-16 more where dy is float32
"""
import math

import pytest
import torch

import kept_ref as ref
import moe_ref
import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
SHAPES = [(1, 1), (1, 32), (3, 7), (5, 33), (2, 31), (64, 64), (17, 100), (130, 257), (9, 2048), (700, 130), (3, 8200), (1, 70001)]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def wide_range(R, C, g, dtype):
    """Values whose blocks differ by powers of ten, zeros, and ties among them."""
    x = torch.randn(R, C, generator=g) * 10.0**torch.randint(-6, 7, (R, 1), generator=g) * torch.rand(R, C, generator=g)**3
    x[torch.rand(R, C, generator=g) < 0.1] = 0.0
    whole = torch.randint(-255, 256, (R, C), generator=g) * 0.5   # halves of a step of 1 where a block's largest is below 128
    return torch.where(torch.rand(R, 1, generator=g) < 0.3, whole, x).to(dtype)


def same(got, want):
    """Equal values, NaN in the same places."""
    got, want = got.detach().cpu().double(), want.double()
    return got.shape == want.shape and bool(((got == want) | (got.isnan() & want.isnan())).all())


def near(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = (got - want).abs() > bound
    assert not bad.any() and not got.isnan().any(), (what, int(bad.sum()), float((got - want).abs().max()))


def strided(t, pad, at):
    """The same values in rows `pad` elements longer that begin at element `at`; NaN around them."""
    w = torch.full((t.shape[0], t.shape[1] + pad), math.nan, dtype=t.dtype)
    w[:, at:at + t.shape[1]] = t
    return w.to(DEV)[:, at:at + t.shape[1]]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_keep_and_restore(shape, dtype):
    x = wide_range(*shape, gen(sum(shape)), dtype)
    codes, scales = ref.keep(x)
    for xd in (x.to(DEV), strided(x, 5, 3), strided(x, 8, 8)):
        kept = P.keep8(xd)
        assert kept.cols == shape[1]
        assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.scales.cpu(), scales)
        for out in (BF, F32):
            assert same(P.restore8(kept, dtype=out), ref.restore(codes, scales, shape[1]))
    assert P.restore8(kept).dtype == BF


def test_edges_of_the_scale():
    """The largest and smallest numbers, subnormal ones, a block's largest on either side of 127.5 s, infinities and NaN."""
    big, inf, nan = torch.finfo(F32).max, math.inf, math.nan
    rows = [[big, -big, 1.0], [2.0**-126, 2.0**-149, -2.0**-133], [2.0**-120, 2.0**-127, 2.0**-126], [0.0, -0.0, 0.0],
            [127.5, 126.5, 0.5], [127.50001, 1.0, 3.0], [255.0, 1.0, -1.0], [255.00003, 1.0, 3.0], [inf, 1.0, -2.0], [nan, 5.0, -inf],
            [-inf, inf, nan], [127.0, -127.5, 1.5], [2.0**-119 * 127.5, 2.0**-119, 2.0**-126]]
    x = torch.zeros(len(rows), 40)
    x[:, 30:33] = torch.tensor(rows)   # across the end of a block
    x[:, :3] = torch.tensor(rows)
    codes, scales = ref.keep(x)
    kept = P.keep8(x.to(DEV))
    assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.scales.cpu(), scales)
    want = ref.restore(codes, scales, 40)
    assert same(P.restore8(kept), want) and same(P.restore8(kept, dtype=F32), want)
    finite = x.double().isfinite()
    step = torch.exp2(scales.double() - 127).repeat_interleave(32, 1)[:, :40]
    top = x.abs() > 127.5 * 2.0**121   # (kept as 127 steps of the largest scale)
    assert bool(((want - x.double()).abs() <= torch.where(top, 1.0, 0.5) * step)[finite].all())
    assert bool(want[~finite].isnan().all())


def test_every_code_and_scale_is_restored():
    codes = torch.arange(-128, 128).repeat(254).to(torch.int8).view(254, 256)
    scales = torch.arange(1, 255).to(torch.uint8)[:, None].expand(254, 8).contiguous()
    kept = P.Kept8(codes.to(DEV), scales.to(DEV), 256)
    want = ref.restore(codes, scales, 256)
    big = want.abs() > torch.finfo(F32).max   # (scales that keep8 never makes)
    for dtype in (BF, F32):
        assert same(P.restore8(kept, dtype=dtype), torch.where(big, want.sign() * math.inf, want))


KINDS = ["relu", "silu", "gelu_tanh"]
ACTS = [(1, 1), (2, 33), (70, 64), (33, 130), (9, 2765), (300, 256)]


def _act_inputs(R, C, dtype, seed):
    g = gen(seed)
    x, u, da = (torch.randn(R, C, generator=g) * k for k in (3.0, 1.0, 1e-3))
    x[torch.rand(R, C, generator=g) < 0.05] *= 30     # far into both tails
    x[torch.rand(R, C, generator=g) < 0.05] = 0.0
    return x.to(dtype), u.to(dtype), da.to(dtype)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("types", [(BF, BF), (F32, F32), (BF, F32), (F32, BF)], ids=str)
@pytest.mark.parametrize("shape", ACTS, ids=str)
def test_activation(shape, types, kind, gated):
    dtype, out = types
    x, u, da = _act_inputs(*shape, dtype, sum(shape))
    u = u if gated else None
    half = ref.UBF if out == BF else ref.U32

    def check(a, g, v, what):
        f, _, _ = ref.act(g, kind)
        e, _ = ref.act_bound(g, kind)
        v = torch.ones_like(g) if v is None else v
        want = f * v
        near(a, want, (half + 2 * ref.U32) * want.abs() + 1.01 * e * v.abs() + 1e-38, what)

    for xd, ud in ((x.to(DEV), u if u is None else u.to(DEV)), (strided(x, 3, 1), u if u is None else strided(u, 16, 8))):
        a = P.expert_act(xd, ud, kind=kind, dtype=out)
        assert a.dtype == out
        check(a, x.double(), None if u is None else u.double(), "a")
        again, kept = P.expert_act(xd, ud, kind=kind, dtype=out, keep=True)
        assert torch.equal(a, again)
        for k, v in zip(kept, (x, u)):
            if v is None:
                assert k is None
            else:
                codes, scales = ref.keep(v)
                assert torch.equal(k.codes.cpu(), codes) and torch.equal(k.scales.cpu(), scales)
    g8 = ref.restore(*ref.keep(x), shape[1])
    u8 = None if u is None else ref.restore(*ref.keep(u), shape[1])
    for dad in (da.to(DEV), strided(da, 7, 3)):
        a, dg, du = P.expert_act_backward(dad, kept, kind=kind, dtype=out)
        check(a, g8, u8, "a of the kept values")
        f, df, _ = ref.act(g8, kind)
        ef, edf = ref.act_bound(g8, kind)
        d, v = da.double(), torch.ones_like(g8) if u8 is None else u8
        near(dg, d * v * df, (half + 4 * ref.U32) * (d * v * df).abs() + 1.01 * edf * (d * v).abs() + 1e-38, "dg")
        assert (du is None) == (u8 is None)
        if gated:
            near(du, d * f, (half + 2 * ref.U32) * (d * f).abs() + 1.01 * ef * d.abs() + 1e-38, "du")
        none, dg2, du2 = P.expert_act_backward(dad, kept, kind=kind, dtype=out, again=False)
        assert none is None and torch.equal(dg2, dg) and (du is None or torch.equal(du2, du))


@pytest.mark.parametrize("kind", KINDS)
def test_activation_gradient_against_differences(kind):
    """dg and du of float32 rows against differences of the definition at the kept values."""
    x, u, da = _act_inputs(40, 96, F32, 5)
    x[x.abs() < 0.3] = 0.5   # (relu has no derivative at 0)
    da = da * 1e3
    _, kept = P.expert_act(x.to(DEV), u.to(DEV), kind=kind, keep=True)
    _, dg, du = P.expert_act_backward(da.to(DEV), kept, kind=kind)
    g8, u8 = (P.restore8(k, dtype=F32).cpu().double() for k in kept)
    h = 1e-4
    away = (g8.abs() > h) | (kind != "relu")
    fd = (ref.act(g8 + h, kind)[0] - ref.act(g8 - h, kind)[0]) / (2 * h)
    # a central difference is off by h^2 / 6 of the third derivative (below 4 for each f), float32 by some 1e-5
    assert bool(((dg.cpu().double() - da.double() * u8 * fd).abs() <= (1e-7 + 2e-5) * (da.double() * u8).abs() + 1e-9)[away].all())
    assert bool(((du.cpu().double() - da.double() * ref.act(g8, kind)[0]).abs() <= 2e-5 * (da.double() * (1 + g8.abs())).abs()).all())


@pytest.mark.parametrize("kind", KINDS)
def test_activation_of_extreme_values(kind):
    inf, nan = math.inf, math.nan
    x = torch.tensor([[-inf, inf, nan, 0.0, -0.0, 1e30, -1e30, 3e38, -3e38, 1e-40, -100.0, 100.0, -88.0, 88.0]])
    f, df, _ = ref.act(x.double(), kind)
    a, kept = P.expert_act(x.to(DEV), kind=kind, keep=True)
    got = a.cpu().double()
    assert bool((got.isnan() == x.isnan()).all())
    ok = ~x.isnan()
    assert bool((((got - f).abs() <= 1e-4 * f.abs() + 1e-36) | (got == f))[ok].all())
    codes = P.keep8(x.to(DEV)).codes.cpu()[0, :3]
    assert codes.tolist() == [-128] * 3
    # each value in a block of its own; what was infinite is NaN, and so is its gradient
    alone = torch.zeros(1, 14 * 32)
    alone[0, ::32] = x[0]
    _, kept = P.expert_act(alone.to(DEV), kind=kind, keep=True)
    _, dg, _ = P.expert_act_backward(torch.ones_like(alone).to(DEV), kept, kind=kind)
    dg, g8 = dg.cpu().double()[0, ::32], P.restore8(kept[0], dtype=F32).cpu().double()[0, ::32]
    assert bool((dg.isnan() == g8.isnan()).all()) and bool((g8.isnan() == ~x[0].isfinite()).all())
    _, df, _ = ref.act(g8, kind)
    ok = ~g8.isnan()
    assert bool(((dg - df).abs() <= 1e-4 * df.abs() + 1e-30)[ok].all())


# T, E, k, n, m: tiles through registers and straight to LDS, odd widths, experts without rows
GRADS = [(1, 2, 1, 8, 8), (3, 4, 2, 33, 17), (40, 3, 2, 128, 200), (420, 8, 2, 1024, 264), (300, 70, 2, 130, 64),
         (500, 4, 1, 1031, 301), (2, 3, 1, 1, 1)]


@pytest.mark.parametrize("dy_type", [BF, F32])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("case", GRADS, ids=lambda c: "x".join(map(str, c)))
def test_weights_gradient_from_kept_rows(case, gather, dy_type):
    T, E, k, n, m = case
    g = gen(T + n)
    experts = moe_ref.draw_experts(T, E, k, g)
    plan = P.expert_rows(experts.to(DEV), E)
    off, row, _ = moe_ref.rows(experts, E)
    x = torch.randn(T if gather else T * k, n, generator=g).to(BF)
    dy = torch.randn(T * k, m, generator=g).to(dy_type)
    kept = P.keep8(x.to(DEV))
    x8 = ref.restore(*ref.keep(x), n)
    want, size = (moe_ref.matmul_grad(x8, dy, off, row, k, gather, absolute=a) for a in (False, True))
    K = int((off[1:] - off[:-1]).max())
    bound = ref.UBF * want.abs() + ((2.0**-16 if dy_type == F32 else 0.0) + (4 * K + 16) * ref.U32) * size + 1e-38
    got = P.expert_matmul_grad(kept, dy.to(DEV), plan, gather=gather)
    near(got, want, bound, case)
    # the same bits as from the restored rows, into an existing strided tensor too
    assert torch.equal(got, P.expert_matmul_grad(P.restore8(kept), dy.to(DEV), plan, gather=gather))
    out = torch.full((E, n + 1, m + 3), 7.0, dtype=BF, device=DEV)
    P.expert_matmul_grad(kept, dy.to(DEV), plan, gather=gather, out=out[:, :n, :m])
    assert torch.equal(out[:, :n, :m], got) and bool((out[:, n:] == 7).all()) and bool((out[:, :, m:] == 7).all())


def test_no_rows():
    e = torch.empty(0, 40, device=DEV, dtype=BF)
    kept = P.keep8(e)
    assert kept.codes.shape == (0, 64) and kept.scales.shape == (0, 2) and P.restore8(kept).shape == (0, 40)
    a, kept = P.expert_act(e, e, keep=True)
    again, dg, du = P.expert_act_backward(a, kept)
    assert again.shape == dg.shape == du.shape == (0, 40)
    plan = P.expert_rows(torch.empty(0, 2, dtype=torch.int32, device=DEV), 3)
    dw = P.expert_matmul_grad(P.keep8(e), torch.empty(0, 24, device=DEV, dtype=BF), plan)
    assert dw.shape == (3, 40, 24) and not dw.any()


def _steps(x, w_gate, w_up, w_down, plan, dout, stream=None):
    """The layer of kept.py's docstring, forward and backward."""
    how = dict(stream=stream)
    g, u = (P.expert_matmul(x, w, plan, gather=True, **how) for w in (w_gate, w_up))
    a, kept = P.expert_act(g, u, keep=True, **how)
    y = P.expert_matmul(a, w_down, plan, dtype=F32, **how)
    kept_x = P.keep8(x, **how)
    dy, _ = P.expert_combine_backward(dout, y, plan, **how)
    da = P.expert_matmul(dout, w_down, plan, gather=True, transpose=True, **how)
    a2, dg, du = P.expert_act_backward(da, kept, **how)
    return (y, P.expert_matmul_grad(a2, dy, plan, **how),
            *(P.expert_matmul_grad(kept_x, d, plan, gather=True, **how) for d in (dg, du)))


def _layer(seed=0, T=300, E=6, d=128, f=192):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x, dout = (torch.randn(T, d, generator=g, device=DEV).to(BF) for _ in range(2))
    ws = [(torch.randn(E, *s, generator=g, device=DEV) * 0.1).to(BF) for s in ((d, f), (d, f), (f, d))]
    experts = torch.rand(T, E, generator=g, device=DEV).argsort(1)[:, :2].int().contiguous()
    return x, *ws, P.expert_rows(experts, E), dout


def test_layer_on_another_stream_and_in_a_graph():
    inputs = _layer()
    want = _steps(*inputs)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        got = _steps(*inputs, stream=stream)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _steps(*inputs)
    with torch.cuda.graph(other):
        outs2 = _steps(*inputs)
    for seed in range(1, 5):
        new = _layer(seed)
        for t, v in zip((*inputs[:4], *inputs[4], inputs[5]), (*new[:4], *new[4], new[5])):
            t.copy_(v)
        want = _steps(*new)
        torch.cuda.synchronize()
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, outs, outs2))


def test_refusals_of_the_binding():
    x = torch.zeros(4, 40, dtype=BF, device=DEV)
    kept = P.keep8(x)
    pair = (kept, kept)
    for err, call in (
            (TypeError, lambda: P.keep8(x.half())), (TypeError, lambda: P.keep8(x.cpu())), (ValueError, lambda: P.keep8(x[0])),
            (ValueError, lambda: P.keep8(x.T)), (ValueError, lambda: P.keep8(x[:1].expand(4, 40))),
            (ValueError, lambda: P.keep8(x[:, :0])),
            (TypeError, lambda: P.restore8(x)), (TypeError, lambda: P.restore8(kept, dtype=torch.float16)),
            (ValueError, lambda: P.restore8(P.Kept8(kept.codes, kept.scales, 30))),
            (ValueError, lambda: P.restore8(P.Kept8(kept.codes, kept.scales, 0))),
            (ValueError, lambda: P.restore8(P.Kept8(kept.codes, kept.scales, 65))),
            (ValueError, lambda: P.restore8(P.Kept8(kept.codes[:3], kept.scales, 40))),
            (TypeError, lambda: P.restore8(P.Kept8(kept.codes.to(torch.uint8), kept.scales, 40))),
            (TypeError, lambda: P.restore8(P.Kept8(kept.codes, kept.scales.cpu(), 40))),
            (ValueError, lambda: P.restore8(P.Kept8(kept.codes.repeat(1, 2)[:, :64], kept.scales, 40))),
            (ValueError, lambda: P.restore8(P.Kept8(torch.zeros(4 * 64 + 1, dtype=torch.int8, device=DEV)[1:].view(4, 64),
                                                    kept.scales, 40))),
            (ValueError, lambda: P.expert_act(x, kind="tanh")), (TypeError, lambda: P.expert_act(x, x.float())),
            (ValueError, lambda: P.expert_act(x, x[:3])), (TypeError, lambda: P.expert_act(x, dtype=torch.float16)),
            (ValueError, lambda: P.expert_act_backward(x[:3], pair)), (ValueError, lambda: P.expert_act_backward(x[:, :39], pair)),
            (TypeError, lambda: P.expert_act_backward(x, (None, kept))), (TypeError, lambda: P.expert_act_backward(x, (kept, x))),
            (ValueError, lambda: P.expert_act_backward(x, (kept, P.keep8(x[:, :33])))),
            (ValueError, lambda: P.expert_act_backward(x, pair, kind="tanh")),
            (RuntimeError, lambda: P.keep8(x.float().requires_grad_())),
            (RuntimeError, lambda: P.expert_act(x, x.clone().requires_grad_())),
            (RuntimeError, lambda: P.expert_act_backward(x.clone().requires_grad_(), pair))):
        with pytest.raises(err):
            call()
    plan = P.expert_rows(torch.zeros(4, 1, dtype=torch.int32, device=DEV), 2)
    for err, call in (
            (ValueError, lambda: P.expert_matmul_grad(kept, x[:3], plan)),
            (ValueError, lambda: P.expert_matmul_grad(P.keep8(x[:3]), x, plan)),
            (TypeError, lambda: P.expert_matmul_grad(kept, x.half(), plan)),
            (ValueError, lambda: P.expert_matmul_grad(kept, x, plan, out=torch.zeros(2, 40, 39, dtype=BF, device=DEV))),
            (TypeError, lambda: P.expert_matmul_grad(kept, x, plan, out=torch.zeros(2, 40, 40, device=DEV)))):
        with pytest.raises(err):
            call()
