"""ll_policy and ll_preference where all logits of a row are far below 0, or a stretch of the vocabulary has no probability at all: legal
inputs, as a softmax does not change under a common shift, and the exponentials' reference is then far from 0 in every tile that has ids."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.conftest import kernels_of, say
from tests.test_gpu_answers import case, check_policy, check_preference, policy_inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def below(N, d, V, nats, seed=0):
    """As `case`, with every logit lower by about `nats` (a column of W_U that all rows meet with one factor)."""
    a, W, ids, g = case(N, d, V, seed=seed)
    a[:, 0], W[:, 0] = -nats / 16, 16.0
    a[::3, 0] = 0.0                                     # rows that stay where they are, beside the others
    a[0, 0] = -nats / 16
    return a, W, ids, g


# (kernel of the first product, ids a workgroup): the last 64 ids of these V hold groups of 16 or 32 that are past the vocabulary; groups of 64,
# tiles of 256 and few rows beside them
@pytest.mark.parametrize("N,d,V,kernel", [
    (16, 136, 2000, "logits_kernel<1, 1>"), (16, 264, 3024, "logits_kernel<1, 1>"), (64, 136, 4000, "logits_kernel<1, 4>"),
    (100, 72, 4000, "logits_kernel<2, 4>"), (40, 136, 10000, "logits_kernel<2, 3>"), (20, 64, 20000, "logits_kernel<4, 2>"),
    (300, 64, 4001, "logits_kernel<4, 4>"), (16, 136, 4096, "logits_kernel<1, 1>"),
    (40, 64, 30000, "others_kernel"), (3, 64, 4000, "few_others_kernel")])
@pytest.mark.parametrize("nats", [96.0, 144.0, 208.0])
def test_rows_far_below(N, d, V, kernel, nats):
    say(f"answers {nats} nats below 0, N={N} d={d} V={V}")
    a, W, ids, g = below(N, d, V, nats)
    A, old, ref, weight = policy_inputs(a, W, ids, g, 1.0)
    dev = [x.to(DEV) for x in (a, W, ids, A)]
    assert any(kernel in name for name in kernels_of(lambda: LL.ll_policy(*dev)))
    check_policy(a, W, ids, A, old, ref, weight, 0.2, 0.2, 0.1, 1.0)
    check_preference(a, W, ids, torch.tensor([0, N // 3, N // 2, N // 2, N], dtype=torch.int32), None, None, 0.1, 0.0, "logistic", False, 1.0)


def test_a_low_temperature_brings_logits_as_far():
    N, d, V = 16, 136, 4000
    say("answers far below 0 by their temperature")
    a, W, ids, g = below(N, d, V, 64.0)
    A, old, ref, weight = policy_inputs(a, W, ids, g, 0.5)
    check_policy(a, W, ids, A, old, ref, weight, 0.2, 0.2, 0.1, 0.5)


@pytest.mark.parametrize("N,V", [(16, 4000), (100, 4000), (20, 20000), (40, 30000), (3, 4000)])
def test_a_stretch_of_the_vocabulary_without_probability(N, V):
    """Ids 1600 to 1727 at minus infinity, or a million nats down, take no part: of the other columns every bit is the same."""
    d = 72
    say(f"answers beside ids without probability N={N} V={V}")
    a, W, ids, g = below(N, d, V, 176.0)
    a[:, 0] = -11.0
    ids = torch.where((ids >= 1600) & (ids < 1728), 5, ids)
    A = torch.randn((N,), generator=g)
    got = []
    for far in (1e5, float("inf")):
        W[1600:1728, 0] = far
        got.append(LL.ll_policy(*[x.to(DEV) for x in (a, W, ids, A)]))
    for x, y in zip(*(g[:2] + (g[2][:, 1:],) for g in got)):
        assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))
        assert torch.isfinite(x[ids.to(DEV) >= 0 if N == 3 else slice(3, None)]).all()
