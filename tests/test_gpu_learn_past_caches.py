"""The products that learn through the lens past the caches: one row block and more of W_U than the Infinity Cache holds."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.conftest import kernels_of, say
from tests.test_gpu_learn import check_distill, check_logp, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
d, V, k = 2048, 70000, 6       # 287 MB, two tiles a workgroup


@pytest.fixture(scope="module")
def case():
    return inputs(250, d, V, k)


@pytest.mark.parametrize("N,row_tiles", [(20, 1), (64, 1), (100, 2), (180, 3), (250, 4)])
def test_against_the_oracle(case, N, row_tiles):
    say(f"past the caches N={N} d={d} V={V}")
    a, W, ids, g = case
    a, ids = a[:N].contiguous(), ids[:N].contiguous()
    _, lse, ent, _ = check_logp(a, W, ids, g, 0.7)
    scores, weight = 3 * torch.randn((N, k), generator=g), torch.rand((N,), generator=g)
    check_distill(a, W, ids, scores, weight, 2.0)
    ca, cW, cids, cs = (x.to(DEV) for x in (a, W, ids, scores))
    found = [n.split("(")[0] for n in kernels_of(lambda: (LL.ll_logp(ca, cW, cids), LL.ll_distill(ca, cW, cids, cs), LL.ll_logp_grad(ca, cW, cids, lse, ent, cs)))]
    assert {n for n in found if "logits_kernel" in n or "back_kernel" in n} == {
        f"ll_learn_logits_kernel<{what}, false, {row_tiles}, true>" for what in (0, 1, 2)} | {f"ll_learn_back_kernel<{row_tiles}, true>"}, found
