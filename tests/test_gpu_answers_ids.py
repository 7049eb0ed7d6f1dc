"""ll_policy and ll_preference with the least and the largest ids that 32 bits hold: rows without a token, on every path."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.conftest import say
from tests.test_gpu_answers import case
from tests.test_gpu_learn import INT_MAX, INT_MIN

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("N,d,V", [(4, 512, 900), (70, 328, 4000), (40, 64, 30000)])
def test_ids_at_the_ends_of_their_type(N, d, V):
    """The others' every bit is as with -1 there."""
    a, W, ids, g = case(N, d, V, seed=13)
    ids = ids.clamp(0, V - 1)
    A, offsets = torch.randn((N,), generator=g).to(DEV), torch.tensor([0, N // 2, N], dtype=torch.int32, device=DEV)
    a, W = a.to(DEV), W.to(DEV)
    at = [1, N - 1]
    got = []
    for values in ((-1, -1), (INT_MIN, INT_MAX), (INT_MIN + 5, -2), (V, INT_MIN + V)):
        say(f"answers with ids {values} N={N}")
        odd = ids.clone()
        odd[at] = torch.tensor(values, dtype=torch.int32)
        odd = odd.to(DEV)
        got.append(LL.ll_policy(a, W, odd, A) + LL.ll_preference(a, W, odd, offsets))
    for other in got[1:]:
        for x, y in zip(got[0], other):
            assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))
    assert torch.isnan(got[0][1][at]).all() and not got[0][0][at].any() and not got[0][2][at].any() and not got[0][6][at].any()
