"""Refusals of the operators' outputs, whatever stream they are called on."""
import pytest
import torch

import paper_2607_19058_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.mark.parametrize("other", [False, True], ids=["current", "other"])
def test_outputs_are_checked_first(other):
    stream = torch.cuda.Stream() if other else None
    plan = P.expert_rows(torch.zeros(4, 1, dtype=torch.int32, device=DEV), 2)
    x, dy = torch.zeros(4, 8, dtype=BF, device=DEV), torch.zeros(4, 16, dtype=BF, device=DEV)
    ids, rows = torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros(4, 8, device=DEV)
    torch.cuda.synchronize()
    for err, out in ((TypeError, torch.zeros(2, 8, 16, dtype=BF)), (TypeError, torch.zeros(2, 8, 16, device=DEV)),
                     (ValueError, torch.zeros(2, 8, 15, dtype=BF, device=DEV)), (ValueError, torch.zeros(3, 8, 16, dtype=BF, device=DEV))):
        with pytest.raises(err):
            P.expert_matmul_grad(x, dy, plan, out=out, stream=stream)
    for err, out in ((TypeError, torch.zeros(5, 8)), (TypeError, torch.zeros(5, 8, dtype=BF, device=DEV)),
                     (ValueError, torch.zeros(4, 8, device=DEV))):
        with pytest.raises(err):
            P.embed_grad(ids, rows, 5, out=out, stream=stream)
    torch.cuda.synchronize()
