"""Gradients of words that no token gives a probability that float16 holds beside the tokens' factors: they keep the accuracy of the others.

A word is rare here where every |G_tv| is below sqrt(T) 2^-31 of its token's factor (include/skew_loss.h). Bounds as in tests/loss_ref.py, but
without what an entry may lose below float16's normal numbers beside its row's factor; instead 2^-39 of its word's largest (half a step of
2^-24, of a largest that is kept as 2^14 or more).
"""
import math

import pytest
import torch

import paper_2607_19058_amd as P
from loss_ref import F16, F16_LOW, U32, UBF, Ref
from test_gpu_loss import inputs, near

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def rare_inputs(T, d, V, tied, every=7, run=(20, 60), far=(16, 24, 28, 32, 40, 56, 70), seed=0):
    """x's first column is 8, and w's first column takes 16 to 70 off the logits of every seventh word and of a run of words."""
    x, w, targets, _, _ = inputs(T, d, V, tied=tied, none=0.05, seed=seed)
    g = torch.Generator(device=DEV).manual_seed(seed + T)
    words = w if tied else w.T
    less = torch.zeros(V, device=DEV)
    at = torch.arange(V, device=DEV)
    these = (at % every == 3) | ((at >= run[0]) & (at < run[1])) if every else torch.ones(V, dtype=torch.bool, device=DEV)
    less[these] = torch.tensor(far, device=DEV, dtype=F32)[torch.randint(0, len(far), (int(these.sum()),), generator=g, device=DEV)]
    words[:, 0] = (-less / 8).to(BF)
    x[:, 0] = 8.0
    common = torch.nonzero(~these).squeeze(1) if every else at[:1]
    there = (targets >= 0) & (targets < V)
    targets[there] = common[targets[there] % common.numel()]
    dloss = torch.rand(T, generator=g, device=DEV) + 0.5
    return x, w, targets, dloss, these


def dw_of(ref, dloss, dlse=None):
    """(dw by words, its bound for rare words, which are rare)"""
    one = torch.where(ref.there, ref.scale * dloss.double(), 0.0)
    both = one + (0.0 if dlse is None else torch.where(ref.there, ref.scale * dlse.double(), 0.0))
    n = torch.arange(one.numel(), device=DEV)
    p = torch.exp(ref.z - ref.lse_all[:, None])
    G = both[:, None] * p
    G[n, ref.y] -= one
    factor = torch.maximum(both.abs(), one.abs())
    share = torch.where(ref.there, G.abs().T / factor.clamp(min=1e-300), 0.0).T
    top = share.amax(0)
    e = ref.ez + ref.e_lse[:, None] + (4 * ref.z.abs() + 16) * U32
    eG = (both.abs())[:, None] * p * e.expm1() + (F16 + 8 * U32) * G.abs() + 2 * F16_LOW * factor[:, None] * top
    Ga = G.abs() + eG
    dw = G.T.contiguous() @ ref.x
    ex = F16_LOW * ref.x.abs().amax(0)
    less = torch.where(factor > 0, factor.max() / factor, 0.0)
    bound = eG.T.contiguous() @ ref.x.abs() + (Ga * less[:, None]).sum(0)[:, None] * ex
    bound = bound + (2 * G.shape[0] + 16) * U32 * (Ga.T.contiguous() @ ref.x.abs())
    return dw, 1.01 * bound + 1.01 * UBF * dw.abs() + 1e-38, top < math.sqrt(G.shape[0]) * 2.0**-31


# (tokens, width, words) with float16 operands: one piece and two, odd sizes, words in copies
CASES = [(600, 1000, 904), (530, 1031, 1001), (4100, 24, 66010), (2100, 33, 8011), (700, 2033, 380)]


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_rare_words_keep_their_gradient(case, tied):
    T, d, V = case
    x, w, targets, dloss, these = rare_inputs(T, d, V, tied)
    ref = Ref(x, w, targets, tied)
    loss, lse = P.head_loss(x, w, targets, tied=tied)
    near(loss, ref.loss, ref.e_loss, "loss")
    g = torch.Generator(device=DEV).manual_seed(9)
    for dlse in (None, torch.rand(T, generator=g, device=DEV) * 0.1):
        dx, bx, dw, bw = ref.backward(dloss, dlse)
        gx, gw = P.head_loss_backward(x, w, targets, lse, dloss, dlse=dlse, tied=tied)
        near(gx, dx, bx, "dx")
        near(gw, dw, bw, "dw")
        want, bound, rare = dw_of(ref, dloss, dlse)
        assert int(rare.sum()) > V // 20 and not rare.all()
        near((gw if tied else gw.T)[rare], want[rare], bound[rare], "dw of rare words")


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("case", [(600, 1000, 904), (4100, 24, 66010)], ids=lambda c: "x".join(map(str, c)))
def test_all_words_but_one_are_rare(case, tied):
    """One word takes all the probability; and with a stride, into an existing tensor."""
    T, d, V = case
    x, w, targets, dloss, _ = rare_inputs(T, d, V, tied, every=0, far=(32, 40, 56, 70))
    (w if tied else w.T)[0, 0] = 0.0
    ref = Ref(x, w, targets, tied)
    _, lse = P.head_loss(x, w, targets, tied=tied)
    want, bound, rare = dw_of(ref, dloss)
    assert int(rare.sum()) > 0.99 * V
    out = torch.full((w.shape[0], w.shape[1] + 3), 7.0, dtype=BF, device=DEV)
    _, gw = P.head_loss_backward(x, w, targets, lse, dloss, tied=tied, out=out[:, 1:-2])
    near((gw if tied else gw.T)[rare], want[rare], bound[rare], "dw of rare words")
    assert bool((out[:, 0] == 7).all()) and bool((out[:, -2:] == 7).all())


@pytest.mark.parametrize("tied", [False, True])
def test_a_rare_word_that_is_a_target(tied):
    """Its entry is its token's whole factor: the word is not rare any more. With dloss far below dlse it still is."""
    T, d, V = 600, 1000, 904
    x, w, targets, dloss, these = rare_inputs(T, d, V, tied, far=(40,))
    v = torch.nonzero(these).squeeze(1)
    targets[5], targets[6] = v[0], v[1]
    ref = Ref(x, w, targets, tied)
    _, lse = P.head_loss(x, w, targets, tied=tied)
    dx, bx, dw, bw = ref.backward(dloss)
    gx, gw = P.head_loss_backward(x, w, targets, lse, dloss, tied=tied)
    near(gx, dx, bx, "dx")
    near(gw, dw, bw, "dw")
    want, bound, rare = dw_of(ref, dloss)
    assert not rare[v[:2]].any() and rare[v[2:]].all()
    near((gw if tied else gw.T)[rare], want[rare], bound[rare], "dw of rare words")
    dlse = torch.ones_like(dloss)
    dloss = dloss * 1e-14
    want, bound, rare = dw_of(ref, dloss, dlse)
    assert rare[v].all()
    _, gw = P.head_loss_backward(x, w, targets, lse, dloss, dlse=dlse, tied=tied)
    near((gw if tied else gw.T)[rare], want[rare], bound[rare], "dw of rare words")


@pytest.mark.parametrize("tied", [False, True])
def test_rare_words_in_graphs(tied):
    """Which words are rare, and how many, differs from replay to replay; two graphs of the same inputs."""
    T, d, V = 600, 1000, 904
    args = rare_inputs(T, d, V, tied)[:4]
    x, w, targets, dloss = args

    def run():
        loss, lse = P.head_loss(x, w, targets, tied=tied)
        return (loss, lse, *P.head_loss_backward(x, w, targets, lse, dloss, tied=tied))
    run()
    torch.cuda.synchronize()
    graphs, outs = (torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()), []
    for graph in graphs:
        with torch.cuda.graph(graph):
            outs.append(run())
    for seed, how in enumerate((dict(every=5), dict(every=100, run=(0, 0)), dict(every=900, run=(0, 0), far=(0,)), dict(every=2))):
        for t, v in zip(args, rare_inputs(T, d, V, tied, seed=seed, **how)):
            t.copy_(v)
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(a, b) for a, b in zip(want, o))


@pytest.mark.parametrize("tied", [False, True])
def test_entries_below_float16s_normal_numbers(tied):
    """A word that is rare for one token alone is kept beside that token's factor, here 1 (kept as 2^13): from 2^-27 of it on with 11 bits, below
    that in steps of 2^-37. A column of x that is zero for the other tokens shows that token's entries."""
    T, d, V = 600, 1000, 904
    x, w, targets, _, _ = inputs(T, d, V, tied=tied, none=0.0)
    words = w if tied else w.T
    less = torch.arange(V, device=DEV) % 27   # p from 2^-10 to 2^-47
    words[:, 0] = (-less / 8).to(BF)
    x[:, 0], x[:, 5], x[7, 0], x[7, 5] = 0.0, 0.0, 8.0, 1.5
    targets[7] = 0
    dloss = torch.ones(T, device=DEV)
    ref = Ref(x, w, targets, tied)
    _, lse = P.head_loss(x, w, targets, tied=tied)
    _, dw = P.head_loss_backward(x, w, targets, lse, dloss, tied=tied)
    G = torch.exp(ref.z[7] - ref.lse_all[7])
    G[0] -= 1
    assert int(((G > 2.0**-28) & (G < 2.0**-27)).sum()) > 5 and int((G.abs() < 2.0**-38).sum()) > 20
    e = (ref.ez[7] + ref.e_lse[7] + (4 * ref.z[7].abs() + 16) * U32).expm1()
    off = (e + 8 * U32) * G.abs() + torch.where(G.abs() >= 2.0**-27, F16 * G.abs(), 2.0**-38)
    got = (dw if tied else dw.T)[:, 5]
    near(got, 1.5 * G, 1.01 * (1.5 * off + UBF * 1.5 * G.abs()) + 1e-37, "dw")
