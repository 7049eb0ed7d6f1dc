"""ll_policy and ll_preference beside infinities and NaN that their documentation allows: references without probability, rows that hold no number."""

import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.conftest import say
from tests.test_gpu_answers import case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


@pytest.mark.parametrize("N", [4, 40])
@pytest.mark.parametrize("form,smoothing", [("logistic", 0.0), ("logistic", 0.25), ("hinge", 0.0), ("square", 0.0)])
def test_an_infinite_reference(N, form, smoothing):
    """A score of plus or minus infinity has the limit of the loss, and where that is flat no gradient; the other pair is as without it."""
    d, V = 64, 300
    a, W, ids, g = case(N, d, V, seed=11)
    ids = ids.clamp(0, V - 1)
    offsets = torch.tensor([0, 1, 2, 3, N], dtype=torch.int32)
    ref = torch.full((N,), -3.0)
    dev = lambda *t: [x.to(DEV) for x in t]  # noqa: E731
    kw = dict(form=form, smoothing=smoothing, beta=0.5)
    clean = LL.ll_preference(*dev(a, W, ids, offsets), ref_logp=ref.to(DEV), **kw)
    for row, value, h in ((0, -INF, INF), (1, -INF, -INF), (0, INF, -INF), (1, INF, INF)):
        say(f"preference {form} {smoothing} at h = {h}, N={N}")
        bad = ref.clone()
        bad[row] = value
        loss, score, logp, grad = LL.ll_preference(*dev(a, W, ids, offsets), ref_logp=bad.to(DEV), **kw)
        alone = LL.ll_preference(*dev(a, W, ids, offsets), ref_logp=bad.to(DEV), **kw, grad=False)
        want = {"logistic": (smoothing if h > 0 else 1 - smoothing) and INF, "hinge": 0.0 if h > 0 else INF, "square": INF}[form]
        assert float(loss[0]) == float(alone[0][0]) == want
        assert float(score[0, row]) == -value and torch.equal(score[0, 1 - row], clean[1][0, 1 - row])
        assert torch.equal(loss[1], clean[0][1]) and torch.equal(score[1], clean[1][1]) and torch.equal(logp, clean[2])
        assert torch.equal(grad[2:], clean[3][2:])
        if form == "hinge" and h > 0 or form == "logistic" and smoothing == 0 and h > 0:
            assert not grad[:2].any()
        elif form != "square":
            assert torch.isfinite(grad[:2]).all() and grad[:2].any()
