"""How often a distillation's gradient is rounded."""
import numpy as np
import pytest
import torch

import oracle.learn_oracle as O
from paper_2604_06483_amd import binding as LL
from tests.conftest import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("N", [300, 70])
def test_rows_whose_reference_moves_are_rounded_no_more_often(N):
    """W_U is the identity, so that the gradient is dz itself: rounded between the products and as the result, by up to 2^-8 of itself each;
    the exponentials of logits up to 61 come from fp32 numbers below 2^7 in powers of two, off by 2^-18 of themselves at most, some of them.
    The lists are 40 nats and more below the rest, so that every row's reference moves."""
    say(f"moved references, N={N}")
    V = 256
    g = torch.Generator().manual_seed(11)
    z = (50 + 11 * torch.rand((N, V), generator=g)).to(torch.bfloat16)
    ids = torch.stack([torch.randperm(V, generator=g)[:3] for _ in range(N)])
    z.scatter_(1, ids, torch.randn((N, 3), generator=g).to(torch.bfloat16))
    scores, weight = torch.randn((N, 3), generator=g), 0.3 + torch.rand((N,), generator=g)
    W = torch.eye(V, dtype=torch.bfloat16)
    _, grad = LL.ll_distill(z.to(DEV), W.to(DEV), ids.to(torch.int32).to(DEV), scores.to(DEV), weight=weight.to(DEV))
    f64 = lambda t: t.double().numpy()
    dz = O.distill(f64(z), f64(W), ids.numpy(), f64(scores), 1.0, f64(weight))[1]
    off = np.abs(f64(grad.cpu()) - dz) / np.abs(dz)
    assert np.max(off) <= (1 + 2.0 ** -8) ** 2 - 1 + 2e-5, float(np.max(off)) * 2 ** 8
