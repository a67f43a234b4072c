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
