"""Training through the lens where something else than the rows is trained, or a row is no number."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from paper_2604_06483_amd import tune
from tests.conftest import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(N, d, V, k, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV)
    return (normal(N, d).to(torch.bfloat16), (0.1 * normal(V, d)).to(torch.bfloat16),
            torch.randint(0, V, (N, k), generator=g, device=DEV, dtype=torch.int32), normal(N, k), torch.rand((N,), generator=g, device=DEV))


@pytest.mark.parametrize("N", [3, 70])
@pytest.mark.parametrize("trained", [True, False])
def test_the_weight_of_a_distillation_gets_its_gradient(N, trained):
    say(f"distill, gradient of the weight, N={N} rows trained={trained}")
    rows, W, ids, scores, weight = inputs(N, 128, 700, 4)
    loss, grad = LL.ll_distill(rows, W, ids, scores, weight=weight, grad=trained)
    rows.requires_grad_(trained)
    weight.requires_grad_()
    out = tune.distill(rows, W, ids, scores, weight=weight)
    assert torch.equal(out.detach(), weight.detach() * loss)
    out.sum().backward()
    assert torch.equal(weight.grad, loss)
    assert torch.equal(rows.grad, grad) if trained else rows.grad is None
