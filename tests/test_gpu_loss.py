"""The head's loss and its gradients on the GPU against their definitions in float64, within the bounds of tests/loss_ref.py."""
import math

import pytest
import torch

import paper_2607_19058_amd as P
from loss_ref import Ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def near(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(((got - want).abs() / bound).nan_to_num(1e9).max()))


def inputs(T, d, V, tied=False, seed=0, learnt=8.0, none=0.1, wide=False):
    g = torch.Generator(device=DEV).manual_seed(seed + 1000 * T + d + V)
    w = (torch.randn(V, d, generator=g, device=DEV) * d**-0.5).to(BF)
    targets = torch.randint(0, V, (T,), generator=g, device=DEV)
    boost = torch.rand(T, 1, generator=g, device=DEV) * learnt
    x = torch.randn(T, d, generator=g, device=DEV) + boost * w[targets].float()
    if wide:   # columns that differ by many powers of two, against each other in x and w
        power = torch.randint(-40, 41, (d,), generator=g, device=DEV).float()
        x, w = torch.ldexp(x, power), torch.ldexp(w.float(), -power).to(BF)
    out = torch.rand(T, generator=g, device=DEV)
    targets[out < none] = -1
    targets[out > 1 - none / 2] = V
    dloss = torch.randn(T, generator=g, device=DEV) / max(T, 1)
    dlse = torch.randn(T, generator=g, device=DEV) * 1e-2 / max(T, 1)
    return x.to(BF), w if tied else w.T.contiguous(), targets, dloss, dlse


def check(x, w, targets, dloss, dlse, tied, scale=1.0, dtype=None, ref=None):
    ref = ref or Ref(x, w, targets, tied, scale)
    loss, lse = P.head_loss(x, w, targets, tied=tied, scale=scale)
    assert loss.dtype == lse.dtype == F32
    near(loss, ref.loss, ref.e_loss, "loss")
    near(lse, ref.lse, ref.e_lse, "lse")
    dx, bx, dw, bw = ref.backward(dloss, dlse, dtype != F32)
    gx, gw = P.head_loss_backward(x, w, targets, lse, dloss, dlse=dlse, tied=tied, scale=scale, dtype=dtype)
    assert gx.dtype == (dtype or BF) and gw.dtype == BF
    near(gx, dx, bx, "dx")
    near(gw, dw, bw, "dw")
    return loss, lse, gx, gw


SMALL = [(1, 1, 1), (1, 8, 8), (1, 64, 1000), (2, 3, 2), (3, 33, 17), (5, 40, 129), (64, 64, 64), (65, 128, 300), (70, 31, 257),
         (130, 256, 512), (257, 40, 1001), (300, 130, 777), (31, 2048, 96), (40, 2000, 264), (1, 1031, 4100),
         (1, 1, 16385), (1, 2048, 16401), (2, 33, 17001), (16, 100, 20003), (17, 100, 20003), (9, 523, 16388),
         (512, 24, 70), (513, 8, 8), (515, 1, 9), (530, 33, 129), (700, 31, 257), (600, 200, 1001)]
# more than 512 tokens and 2^29 of tokens * d * vocab: float16 operands of the gradients' products
FLOAT16 = [(513, 1, 1046600), (530, 33, 30701), (513, 1024, 1024), (700, 2033, 377), (4000, 513, 263), (40000, 1031, 15), (600, 1000, 901)]


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("case", SMALL, ids=lambda c: "x".join(map(str, c)))
def test_small(case, tied):
    x, w, targets, dloss, dlse = inputs(*case, tied=tied, none=0.1 if case[0] > 2 else 0.0)
    first = check(x, w, targets, dloss, None, tied)
    again = check(x, w, targets.int(), dloss, None, tied)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    check(x, w, targets, dloss, dlse, tied, scale=0.37, dtype=F32)


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("case", FLOAT16, ids=lambda c: "x".join(map(str, c)))
def test_float16_operands(case, tied):
    x, w, targets, dloss, dlse = inputs(*case, tied=tied)
    check(x, w, targets, dloss, None, tied)
    check(x, w, targets, dloss, dlse, tied, scale=0.37, dtype=F32)


# every tile of the logits, the rows' and the weights' gradients; contractions that several work-groups share
LARGE = [(2048, 64, 8192), (1000, 72, 8200), (520, 512, 3000), (4096, 2048, 512), (2500, 1100, 520), (130, 4096, 2056), (2100, 33, 4999)]


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("case", LARGE, ids=lambda c: "x".join(map(str, c)))
def test_large(case, tied):
    check(*inputs(*case, tied=tied), tied)


@pytest.mark.parametrize("tied", [False, True])
def test_pieces_of_the_vocabulary(tied):
    """G in two pieces, the second one ragged; w's copy in two pieces (forward); more rows than a forward launch takes."""
    check(*inputs(4100, 24, 66010, tied=tied), tied)
    x, w, targets, dloss, dlse = inputs(5, 4097, 66001, tied=tied, none=0.0)
    check(x, w, targets, dloss, dlse, tied)
    check(*inputs(16500, 16, 301, tied=tied), tied)
    check(*inputs(33000, 9, 40, tied=tied), tied)


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("T", [1, 16, 17, 33, 150, 600])
def test_strides_and_existing_outputs(T, tied):
    d, V = (72, 520) if T < 600 else (1000, 904)   # (float16 operands)
    x, w, targets, dloss, dlse = inputs(T, d, V, tied=tied, none=0.1 if T > 1 else 0.0)
    want = check(x, w, targets, dloss, dlse, tied)
    for pad, at in ((8, 8), (16, 0), (3, 1), (5, 4)):
        xs = torch.full((T, d + pad), math.nan, dtype=BF, device=DEV)
        ws = torch.full((w.shape[0], w.shape[1] + pad), math.nan, dtype=BF, device=DEV)
        xs[:, at:at + d], ws[:, at:at + w.shape[1]] = x, w
        xv, wv = xs[:, at:at + d], ws[:, at:at + w.shape[1]]
        loss, lse = P.head_loss(xv, wv, targets, tied=tied)
        out = torch.full((w.shape[0] + 1, w.shape[1] + pad), 7.0, dtype=BF, device=DEV)
        view = out[:-1, at:at + w.shape[1]]
        dx, dw = P.head_loss_backward(xv, wv, targets, lse, dloss, dlse=dlse, tied=tied, out=view)
        assert dw is view
        for a, b in zip(want, (loss, lse, dx, view)):
            assert torch.equal(a, b)
        view.fill_(7.0)
        assert bool((out == 7.0).all())


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("T", [40, 140, 600])
def test_rows_that_are_no_token(T, tied):
    d, V = (64, 300) if T < 600 else (1000, 904)
    x, w, targets, dloss, dlse = inputs(T, d, V, tied=tied, none=0.3)
    targets[3], targets[4], targets[5] = -2**40, 2**40, 2**32   # (2^32 is 0 in 32 bits)
    there = (targets >= 0) & (targets < V)
    loss, lse, dx, dw = check(x, w, targets, dloss, dlse, tied)
    assert not loss[~there].any() and not lse[~there].any() and not dx[~there].any()
    x2, dl2, ds2 = x.clone(), dloss.clone(), dlse.clone()
    x2[~there], dl2[~there], ds2[~there] = math.nan, math.nan, math.inf
    loss2, lse2 = P.head_loss(x2, w, targets, tied=tied)
    dx2, dw2 = P.head_loss_backward(x2, w, targets, torch.where(there, lse2, math.nan), dl2, dlse=ds2, tied=tied)
    for a, b in ((loss, loss2), (lse, lse2), (dx, dx2), (dw, dw2)):
        assert torch.equal(a, b)
    none = torch.full_like(targets, -1)
    loss, lse = P.head_loss(x2, w, none, tied=tied)
    dx, dw = P.head_loss_backward(x2, w, none, lse, dloss, tied=tied)
    assert not loss.any() and not lse.any() and not dx.any() and not dw.any()
    e = x[:0]
    loss, lse = P.head_loss(e, w, targets[:0], tied=tied)
    dx, dw = P.head_loss_backward(e, w, targets[:0], lse, loss, tied=tied)
    assert loss.shape == lse.shape == (0,) and dx.shape == (0, d) and dw.shape == w.shape and not dw.any()


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("T", [50, 200, 600])
def test_ranges(T, tied):
    """Columns of very different size, large logits, certain tokens, gradients from 1e-30 to 1e30, zeros."""
    d, V = (72, 400) if T < 600 else (1000, 904)
    x, w, targets, dloss, dlse = inputs(T, d, V, tied=tied, wide=True)
    check(x, w, targets, dloss, dlse, tied)
    x, w, targets, dloss, dlse = inputs(T, d, V, tied=tied, learnt=60.0)
    check(x, w, targets, dloss, None, tied)
    check(x, w, targets, dloss, None, tied, scale=20.0)
    check(x, w, targets, dloss * 1e-30, dlse * 1e-30, tied)
    check(x, w, targets, dloss * 1e30, None, tied)
    far = 10.0**torch.linspace(-30, 0, T, device=DEV)   # tokens whose weights differ by as much: each row of dx has its own power of two
    check(x, w, targets, dloss * far, None, tied)
    check(x, w, targets, dloss * far, dlse * far.flip(0), tied, dtype=F32)
    check(x, w, targets, torch.zeros_like(dloss), dlse, tied)
    check(x, w, targets, torch.zeros_like(dloss), None, tied)
    check(torch.zeros_like(x), w, targets, dloss, None, tied)
    check(x, torch.zeros_like(w), targets, dloss, None, tied)
    check((x * 1e-18).to(BF), (w * 1e-18).to(BF), targets, dloss, None, tied, scale=1e30)


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("T", [20, 80, 600])
def test_what_is_not_finite_reaches_its_own_rows_alone(T, tied):
    d, V = (64, 200) if T < 600 else (1000, 904)
    x, w, targets, dloss, dlse = inputs(T, d, V, tied=tied, none=0.0)
    want = check(x, w, targets, dloss, None, tied)
    x2 = x.clone()
    x2[7, 3], x2[9, 5] = math.nan, math.inf
    loss, lse = P.head_loss(x2, w, targets, tied=tied)
    ok = torch.ones(T, dtype=torch.bool, device=DEV)
    ok[[7, 9]] = False
    assert torch.equal(loss[ok], want[0][ok]) and torch.equal(lse[ok], want[1][ok])
    assert bool(loss[~ok].isnan().all()) and bool(lse[~ok].isnan().all())
    dx, dw = P.head_loss_backward(x2, w, targets, lse, dloss, tied=tied)
    assert torch.equal(dx[ok], want[2][ok]) and bool(dx[~ok].isnan().all()) and bool(dw.isnan().all())
    # a word that is infinitely unlikely: rows of w that are -inf where x is positive
    x3 = x.abs() + 0.1
    w3 = w.clone()
    (w3 if tied else w3.T)[17] = -math.inf
    t3 = torch.where(targets == 17, 16, targets)
    loss, lse = P.head_loss(x3, w3, t3, tied=tied)
    keep = torch.arange(V, device=DEV) != 17
    less = (w3[keep] if tied else w3[:, keep]).contiguous()
    ref = Ref(x3, less, torch.where(t3 > 17, t3 - 1, t3), tied)
    near(loss, ref.loss, ref.e_loss, "loss")
    near(lse, ref.lse, ref.e_lse, "lse")


@pytest.mark.parametrize("tied", [False, True])
def test_float16_below_its_normal_numbers(tied):
    """One column of x is zero but for a token whose factor is 2^-30 of the largest: its entry is kept as 2^-16 or a little more, with half
    steps of 2^-25, 2^-9 of it; G and the result are off by 2^-11 and 2^-8 more."""
    x, w, targets, dloss, _ = inputs(600, 1000, 904, tied=tied, none=0.0)
    dloss = torch.full_like(dloss, 1.0)
    x[:, 5], x[7, 5], dloss[7] = 0.0, 1.5, 2.0**-30
    ref = Ref(x, w, targets, tied)
    _, lse = P.head_loss(x, w, targets, tied=tied)
    _, dw = P.head_loss_backward(x, w, targets, lse, dloss, tied=tied)
    _, _, want, _ = ref.backward(dloss)
    got, want = (t[:, 5] if tied else t[5] for t in (dw.double(), want))
    assert float(want.abs().max()) > 0
    error = (got - want).abs() / want.abs()
    assert float(error.max()) <= 2.0**-9 + 2.0**-11 + 2.0**-8 + 1e-4   # (and float32's errors of the logits)


@pytest.mark.parametrize("tied", [False, True])
def test_gradients_against_differences(tied):
    """sum_t dloss_t loss_t + dlse_t lse_t of the definition moves by <dx, step> and <dw, step>."""
    T, d, V = 60, 48, 130
    x, w, targets, dloss, dlse = inputs(T, d, V, tied=tied)
    dloss, dlse = dloss * T, dlse * T * 100
    _, lse = P.head_loss(x, w, targets, tied=tied, scale=0.8)
    dx, dw = P.head_loss_backward(x, w, targets, lse, dloss, dlse=dlse, tied=tied, scale=0.8, dtype=F32)

    def total(x, w):
        r = Ref(x, w, targets, tied, 0.8)
        return (dloss.double() * r.loss + dlse.double() * r.lse).sum()
    g = torch.Generator(device=DEV).manual_seed(3)
    for _ in range(4):
        sx, sw = (torch.randn(t.shape, generator=g, device=DEV).double() for t in (x, w))
        h = 1e-5
        fx = (total(x.double() + h * sx, w.double()) - total(x.double() - h * sx, w.double())) / (2 * h)
        fw = (total(x.double(), w.double() + h * sw) - total(x.double(), w.double() - h * sw)) / (2 * h)
        # entries are off by 2^-11 and (w) 2^-8 of their size, at random signs; differences by some 1e-8
        assert abs(float((dx.double() * sx).sum() - fx)) <= 2.0**-8 * float((dx.double() * sx).norm()) + 1e-6
        assert abs(float((dw.double() * sw).sum() - fw)) <= 2.0**-6 * float((dw.double() * sw).norm()) + 1e-6


@pytest.mark.parametrize("T, step", [(600, 2.0**-11), (100, 2.0**-16)])
def test_rows_gradient_is_not_rounded_to_bf16(T, step):
    """float32 dx. Entries of G are off by `step` at most each (float16, or what two bf16 numbers leave out), at random signs, which the
    norm of the difference shows: below that of what their sizes add up to in squares, and what float32's sums (2 u a term, some
    thousand of them at random signs: 2^-17) leave."""
    x, w, targets, dloss, _ = inputs(T, 256, 5000, none=0.0)   # (600 tokens: 2^29.5)
    ref = Ref(x, w, targets)
    dx, _, _, _ = ref.backward(dloss)
    _, lse = P.head_loss(x, w, targets)
    got, _ = P.head_loss_backward(x, w, targets, lse, dloss, dtype=F32)
    G = torch.exp(ref.z - ref.lse[:, None])
    G[torch.arange(T, device=DEV), targets] -= 1
    G *= dloss.double()[:, None]
    size = ((G**2) @ (ref.w**2)).sum().sqrt()
    assert float((got.double() - dx).norm()) <= (step + 2.0**-17) * float(size)


def _all(x, w, targets, dloss, dlse, tied, stream=None):
    loss, lse = P.head_loss(x, w, targets, tied=tied, stream=stream)
    return (loss, lse, *P.head_loss_backward(x, w, targets, lse, dloss, dlse=dlse, tied=tied, stream=stream))


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("case", [(300, 64, 520), (90, 33, 301), (600, 1000, 904), (601, 999, 905)], ids=str)
def test_other_streams_and_graphs(case, tied):
    args = inputs(*case, tied=tied)
    want = _all(*args, tied)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        got = _all(*args, tied, stream=stream)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    graphs = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    outs = []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(_all(*args, tied))
    for seed in range(1, 5):
        for t, v in zip(args, inputs(*case, tied=tied, seed=seed)):
            t.copy_(v)
        want = _all(*args, tied)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(a, b) for a, b in zip(want, o))


def test_refusals_of_the_binding():
    x, w, targets, dloss, dlse = inputs(20, 64, 100)
    loss, lse = P.head_loss(x, w, targets)
    back = P.head_loss_backward
    for err, call in (
            (TypeError, lambda: P.head_loss(x.float(), w, targets)), (TypeError, lambda: P.head_loss(x, w.half(), targets)),
            (TypeError, lambda: P.head_loss(x, w, targets.float())), (TypeError, lambda: P.head_loss(x.cpu(), w, targets)),
            (TypeError, lambda: P.head_loss(x, w.cpu(), targets)), (TypeError, lambda: P.head_loss(x, w, targets.cpu())),
            (ValueError, lambda: P.head_loss(x, w, targets[:19])), (ValueError, lambda: P.head_loss(x, w, targets[:, None])),
            (ValueError, lambda: P.head_loss(x[0], w, targets)), (ValueError, lambda: P.head_loss(x[:, :63], w, targets)),
            (ValueError, lambda: P.head_loss(x, w, targets, tied=True)), (ValueError, lambda: P.head_loss(x, w.T, targets, tied=True)),
            (ValueError, lambda: P.head_loss(x, w[:, :0], targets)), (ValueError, lambda: P.head_loss(x[:1].expand(20, 64), w, targets)),
            (ValueError, lambda: P.head_loss(x, w, targets.repeat(2)[::2])),
            *((ValueError, lambda s=s: P.head_loss(x, w, targets, scale=s)) for s in (0.0, -1.0, math.nan, math.inf, 1e31)),
            (RuntimeError, lambda: P.head_loss(x.clone().requires_grad_(), w, targets)),
            (RuntimeError, lambda: P.head_loss(x, w.clone().requires_grad_(), targets)),
            (RuntimeError, lambda: back(x, w, targets, lse, dloss.clone().requires_grad_())),
            (ValueError, lambda: back(x, w, targets, lse[:19], dloss)), (ValueError, lambda: back(x, w, targets, lse, dloss[:19])),
            (ValueError, lambda: back(x, w, targets, lse, dloss, dlse=dlse[:19])), (TypeError, lambda: back(x, w, targets, lse, dloss.to(BF))),
            (ValueError, lambda: back(x, w, targets, lse, dloss.repeat(2)[::2])), (TypeError, lambda: back(x, w, targets, lse.cpu(), dloss)),
            (TypeError, lambda: back(x, w, targets, lse, dloss, dtype=torch.float16)),
            (ValueError, lambda: back(x, w, targets, lse, dloss, out=torch.empty(64, 99, dtype=BF, device=DEV))),
            (ValueError, lambda: back(x, w, targets, lse, dloss, out=torch.empty(100, 64, dtype=BF, device=DEV).T)),
            (TypeError, lambda: back(x, w, targets, lse, dloss, out=torch.empty(64, 100, device=DEV)))):
        with pytest.raises(err):
            call()
