"""tune.preference with a weight of any rank, as the call takes it (no GPU needed)."""
import pytest
import torch

from paper_2604_06483_amd import tune
from tests.test_tune_answers_host import OFFSETS, calls, inputs, plain_preference  # noqa: F401


@pytest.mark.parametrize("size", [(2,), (2, 1), (1, 2)])
def test_weights_of_any_rank(size, monkeypatch):
    """One loss a pair, and the weight's gradient in the weight's shape."""
    monkeypatch.setattr(tune.LL, "ll_preference", lambda *a, weight, **k: plain_preference(*a, weight=weight.reshape(-1), **k))
    rows, W, ids, _, _ = inputs()
    weight = torch.tensor([0.7, 0.0]).reshape(size).requires_grad_()
    loss, _, _ = tune.preference(rows.requires_grad_(), W, ids, OFFSETS, weight=weight)
    want, _, _, grad = plain_preference(rows, W, ids, OFFSETS, weight=weight.reshape(-1))
    assert loss.shape == (2,) and torch.equal(loss.detach(), torch.tensor([0.7, 0.0]) * want)
    loss.sum().backward()
    assert torch.equal(weight.grad, want.reshape(size)) and torch.equal(rows.grad, grad)
