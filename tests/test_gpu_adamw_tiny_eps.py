"""ll_adamw with an eps whose reciprocal 32 bits do not hold: elements that never had a gradient stay where they are."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.conftest import say
from tests.test_gpu_adamw import BF16, F32, Problem, check_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("param", [F32, BF16])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1e-38, 1e-12])
def test_elements_without_a_gradient(param, eight, eps):
    """0 / (0 + eps) is 0 whatever eps; those with a gradient have their quotient."""
    say(f"adamw eps={eps} {param} eight={eight}")
    q = Problem([(1000,)], param=param, eight=eight, seed=15)
    zero = torch.arange(1000) % 3 == 0
    zero[512:768] = True                                  # (a block of 8-bit states that has none)
    for x in (q.g, q.m, q.v):
        x[0][zero] = 0.0
    for x in (q.dg, q.dm, q.dv):
        x[0].view(torch.uint8).view(1000, -1)[zero.to(x[0].device)] = 0
    before = q.dp[0].clone()
    LL.ll_adamw(q.list, 3, rate=1e-2, eps=eps, decay=0.0, seed=11)
    assert torch.equal(q.dp[0][zero.to(before.device)], before[zero.to(before.device)])
    check_step(q, eps=eps, decay=0.0, ran=True)
