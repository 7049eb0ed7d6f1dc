"""tune.preference with a column of weights, as the binding takes it."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from paper_2604_06483_amd import tune
from tests.conftest import say
from tests.test_gpu_tune_answers import answers

pytestmark = pytest.mark.gpu


def test_a_column_of_weights():
    say("preference under autograd, weights [2, 1]")
    rows, W, ids, g = answers(20, 64, 300)
    offsets = torch.tensor([0, 4, 9, 12, 20], dtype=torch.int32, device=rows.device)
    weight = torch.tensor([[0.5], [2.0]], device=rows.device, requires_grad=True)
    leaf = rows.clone().requires_grad_()
    loss = tune.preference(leaf, W, ids, offsets, weight=weight)[0]
    loss.sum().backward()
    want = LL.ll_preference(rows, W, ids, offsets, weight=weight.detach().reshape(-1))
    assert torch.equal(loss.detach(), weight.detach().reshape(-1) * want[0]) and torch.equal(weight.grad, want[0][:, None]) and torch.equal(leaf.grad, want[3])
