"""ll_policy: a row that holds no number has no loss that is one, whatever its advantage and with or without a sampling policy."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.conftest import say
from tests.test_gpu_answers import case, policy_inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("N,d,V", [(4, 512, 900), (70, 328, 1000), (40, 64, 30000)])
@pytest.mark.parametrize("on_policy", [False, True])
@pytest.mark.parametrize("advantage", [0.0, 1.0, -1.0])
def test_policy_of_a_row_without_a_number(N, d, V, on_policy, advantage):
    say(f"policy, NaN row N={N} on policy {on_policy} advantage {advantage}")
    a, W, ids, g = case(N, d, V, seed=12)
    ids = ids.clamp(0, V - 1)
    A, old, _, weight = policy_inputs(a, W, ids, g, 1.0)
    A[N - 1], weight[N - 1] = advantage, 1.0
    for value in (float("nan"), float("inf")):
        b = a.clone()
        b[N - 1, 3] = value
        dev = lambda *t: [x.to(DEV) for x in t]  # noqa: E731
        old_ = None if on_policy else old.to(DEV)
        clean, dirty = LL.ll_policy(*dev(a, W, ids, A), old_), LL.ll_policy(*dev(b, W, ids, A), old_)
        alone = LL.ll_policy(*dev(b, W, ids, A), old_, grad=False)
        for x, y in zip(clean, dirty):
            assert torch.equal(x[:-1], y[:-1]) and torch.isnan(y[-1:]).all()
        assert torch.isnan(alone[0][-1]) and torch.isnan(alone[1][-1]) and not torch.isnan(alone[0][:-1]).any()
        # of weight 0 it passes nothing on; without a token it takes no part
        weight[N - 1] = 0.0
        assert not LL.ll_policy(*dev(b, W, ids, A), old_, weight=weight.to(DEV))[2][-1].any()
        none = ids.clone()
        none[N - 1] = -1
        loss, logp, grad = LL.ll_policy(*dev(b, W, none, A), old_)
        assert float(loss[-1]) == 0.0 and torch.isnan(logp[-1]) and not grad[-1].any()
