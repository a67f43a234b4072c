"""Routing where values are extreme, not finite or nearly alike, against the formulas in float64."""
import math

import pytest
import torch

import moe_ref as ref
import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = math.inf, math.nan


# ---- logits that are not finite, softmax with a bias -----------------------------------------------
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("E", [8, 64, 128, 256, 512, 1024])
def test_nonfinite_logits_show_with_a_bias(E, renormalize):
    """Such an expert is chosen first and the weights are NaN; the others' scores have no value, so they follow by
    their bias, ties by index; closed experts stay closed. Rows beside it are as without it."""
    g = torch.Generator().manual_seed(E)
    logits = torch.randn(6, E, generator=g)
    logits[0, 5], logits[1, 6], logits[2, 7], logits[2, 3] = INF, NAN, NAN, INF
    logits[3, :] = -INF
    logits[3, 2] = NAN
    bias = torch.zeros(E)
    bias[4] = 0.125
    w, e = P.route(logits.to(DEV), 3, bias=bias.to(DEV), renormalize=renormalize)
    assert e.cpu()[:4].tolist() == [[5, 4, 0], [6, 4, 0], [3, 7, 4], [2, -1, -1]]
    w = w.cpu()
    assert w[:3].isnan().all() and w[3, 0].isnan()
    alone, chosen = P.route(logits[4:].to(DEV), 3, bias=bias.to(DEV), renormalize=renormalize)
    assert torch.equal(w[4:], alone.cpu()) and torch.equal(e[4:], chosen) and alone.isfinite().all()


def test_nonfinite_logits_show_with_groups():
    logits = torch.zeros(2, 16)
    logits[0, 13], logits[1, 9] = INF, NAN
    w, e = P.route(logits.to(DEV), 2, bias=torch.zeros(16, device=DEV), groups=4, top_groups=1, group_sum=2)
    assert e.cpu().tolist() == [[13, 12], [9, 8]] and w.isnan().all()


def test_one_infinite_logit_of_eight():
    l = torch.tensor([[0.0, 1.0, 2.0, 3.0, 1.0, INF, 0.0, 2.0]])
    w, e = P.route(l.to(DEV), 2, bias=torch.zeros(8, device=DEV))
    assert e.cpu().tolist() == [[5, 0]] and w.isnan().all()


# ---- weights of sigmoid scores that are small ------------------------------------------------------
SMALL = [[-90.0, -91.0, -95.0, -200.0], [-88.5, -89.5, -300.0, -89.0], [-3e38, -3e38, -3.2e38, -3e38], [5.0, -90.0, -100.0, -2.0],
         [-104.0, -103.0, -120.0, -110.0], [-87.0, -88.0, -87.5, -86.0], [100.0, 90.0, -1.0, -50.0], [-1e4, -10001.0, -1e4, -10002.0]]


@pytest.mark.parametrize("dtype", [F32, BF], ids=["f32", "bf16"])
def test_renormalised_weights_of_small_sigmoid_scores(dtype):
    """w = softmax of log sigmoid(l) over the chosen, of any size; its gradient w_i (1 - s_i) (dw_i - sum_j w_j dw_j).
    An exponential's argument is a difference d of two of the logits, off by |d| half ulps."""
    l = torch.tensor(SMALL).to(dtype)
    k, scale = 3, 1.5
    w, e = P.route(l.to(DEV), k, score="sigmoid", scale=scale)
    e = e.cpu()
    order = torch.argsort(l.float(), dim=1, descending=True, stable=True)[:, :k]
    assert torch.equal(e, order.int())
    x = l.double().gather(1, order)
    log_s = torch.nn.functional.logsigmoid(x)
    want = torch.softmax(log_s, 1)
    d = (x.clamp(max=0) - x.clamp(max=0).max(1, keepdim=True).values).abs().clamp(max=200)
    off = (d + 32) * 2 * ref.U32 * want + 1e-37
    assert ((w.cpu().double() / scale - want).abs() <= off).all(), (w.cpu() / scale, want)
    dw = torch.tensor([[1.0, -2.0, 0.5]]).expand(len(SMALL), k).contiguous()
    got = P.route_backward(l.to(DEV), e.to(DEV), dw.to(DEV), score="sigmoid", scale=scale).cpu().double()
    mean = (want * dw).sum(1, keepdim=True)
    part = scale * want * torch.sigmoid(-x) * (dw - mean)
    full = torch.zeros(l.shape, dtype=torch.float64).scatter_(1, order, part)
    bound = torch.zeros(l.shape, dtype=torch.float64).scatter_(1, order, scale * 3 * (off + 2 * off.sum(1, keepdim=True) * want))
    assert ((got - full).abs() <= bound + full.abs() * (ref.UBF if dtype == BF else ref.U32) + 1e-37).all(), (got, full)


# ---- places without an expert beside a weight that is NaN ------------------------------------------
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_places_without_an_expert_weigh_nothing(score, renormalize):
    l = torch.tensor([[NAN, -INF, -INF, -INF], [-INF, -INF, -INF, 1.0], [-INF] * 4])
    for bias in (None, torch.zeros(4, device=DEV)):
        w, e = P.route(l.to(DEV), 3, score=score, renormalize=renormalize, bias=bias)
        assert e.cpu().tolist() == [[0, -1, -1], [3, -1, -1], [-1, -1, -1]]
        assert w[0, 0].isnan() and not w[:, 1:].any() and not w[2].any()


# ---- choices by scores that are nearly alike --------------------------------------------------------
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_choice_by_scores_of_float32(score):
    """Two experts whose values s + b are 24 half ulps of float32 apart. A float32 evaluation is off by some 12 at most:
    2 of the exponential, 2 or 3 of the sum (1 + small), 1 of the division, 1 of adding the bias, for each of the two."""
    g = torch.Generator().manual_seed(7)
    wrong = 0
    for i in range(96):
        a, b = (-(30 + 30 * torch.rand(2, generator=g))).tolist()   # scores of 1e-13 to 1e-26
        a, b = max(a, b), min(a, b)
        l = torch.tensor([[0.0, a, b]] if score == "softmax" else [[10.0, a, b]])
        x = l.double()[0]
        s = torch.softmax(x, 0) if score == "softmax" else torch.sigmoid(x)
        bias = torch.zeros(3)
        bias[2] = float(s[1] * (1 + (24 if i % 2 else -24) * ref.U32) - s[2])   # the lower score is lifted to the other one
        v = s + bias.double()
        want = 1 if v[1] > v[2] else 2
        if abs(float(v[1] - v[2])) < 23 * ref.U32 * float(v[1]):
            continue   # the bias' own rounding
        _, e = P.route(l.to(DEV), 2, score=score, bias=bias.to(DEV))
        assert int(e[0, 0]) == 0
        wrong += int(e[0, 1]) != want
    assert wrong == 0, wrong
