"""The operators have their backward passes as calls of their own: inputs that autograd would have to follow are refused,
before anything else is looked at, instead of giving results that are cut off from them."""
import pytest
import torch

import paper_2607_19058_amd as P

BF = torch.bfloat16


def calls():
    x, w = torch.zeros(4, 8, dtype=BF), torch.zeros(2, 8, 8, dtype=BF)
    i, f = torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, 1)
    plan = P.ExpertRows(torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), i)
    b = torch.zeros(8)
    return {   # name: (the call, the inputs that can require a gradient)
        "route": (lambda t: P.route(t[0], 2, bias=t[1]), [x, b]),
        "route_backward": (lambda t: P.route_backward(t[0], i, t[1]), [x, f]),
        "expert_matmul": (lambda t: P.expert_matmul(t[0], t[1], plan, scale=t[2]), [x, w, f]),
        "expert_matmul_grad": (lambda t: P.expert_matmul_grad(t[0], t[1], plan), [x, x.clone()]),
        "expert_combine": (lambda t: P.expert_combine(t[0], plan, t[1]), [x, f]),
        "expert_combine_backward": (lambda t: P.expert_combine_backward(t[0], t[1], plan, t[2]), [x, x.clone(), f]),
        "embed": (lambda t: P.embed(i[:, 0], t[0]), [x]),
        "embed_grad": (lambda t: P.embed_grad(i[:, 0], t[0], 5), [x]),
    }


@pytest.mark.parametrize("name", calls())
def test_inputs_that_require_a_gradient_are_refused(name):
    call, tensors = calls()[name]
    for k in range(len(tensors)):
        given = [t.detach().clone().requires_grad_(j == k) for j, t in enumerate(tensors)]
        with pytest.raises(RuntimeError, match="autograd"):
            call(given)
        with torch.no_grad(), pytest.raises(TypeError, match="HIP device"):   # accepted as far as this goes
            call(given)
        with pytest.raises(TypeError, match="HIP device"):
            call([t.detach() for t in given])
