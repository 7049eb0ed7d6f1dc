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


def test_an_unembedding_that_wants_a_gradient():
    """A model's own parameter: fit does not train it, and the calls say that they have no gradient of it."""
    say("W_U that requires a gradient")
    inner, last, gamma, W = tune.synthetic_layers(64, 128, 500, DEV)
    W = torch.nn.Parameter(W)
    result = tune.fit(tune.Translator(128, gamma, 1e-5), inner, last, W, k=4, steps=2)
    assert len(result.losses) == 2 and W.grad is None
    ids = torch.zeros((64, 1), dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError, match="W_U"):
        tune.token_logp(inner, W, ids)
    with pytest.raises(ValueError, match="W_U"):
        tune.distill(inner, W, ids, torch.zeros((64, 1), device=DEV))


def test_a_row_of_weight_zero_adds_nothing_whatever_it_holds():
    say("distill, a row of NaN with weight 0")
    rows, W, ids, scores, weight = inputs(20, 128, 700, 4)
    rows[3, 5], rows[7], weight[3], weight[7] = float("nan"), float("inf"), 0.0, 0.0
    rows.requires_grad_()
    out = tune.distill(rows, W, ids, scores, weight=weight)
    assert torch.isfinite(out).all() and out[3] == 0 and out[7] == 0
    out.sum().backward()
    assert torch.isfinite(rows.grad).all() and not rows.grad[[3, 7]].any()


def test_fit_under_another_default_type():
    say("fit, torch's default type float64")
    inner, last, gamma, W = tune.synthetic_layers(64, 128, 500, DEV)
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float64)
    try:
        wide = tune.fit(tune.Translator(128, gamma, 1e-5), inner, last, W, k=4, steps=2)
    finally:
        torch.set_default_dtype(before)
    assert wide == tune.fit(tune.Translator(128, gamma, 1e-5), inner, last, W, k=4, steps=2)


def test_a_gate_with_the_batch_of_its_rows():
    say("block norm, a gate [B, T, d]")
    B, T, d = 3, 11, 136
    g = torch.Generator(device=DEV).manual_seed(5)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV).to(torch.bfloat16)
    gamma, gx, gn = normal(d), normal(B, T, d), normal(B, T, d)
    leaves = [normal(B, T, d).requires_grad_() for _ in range(3)]
    flat = [t.detach().reshape(B * T, d).clone().requires_grad_() for t in leaves]
    for h, y, gate in (leaves, flat):
        out = tune.block_norm(h, y, gamma, 1e-5, gate=gate, scale=0.5)
        torch.autograd.backward(out, [gx.reshape(h.shape), gn.reshape(h.shape)])
    for a, b in zip(leaves, flat):
        assert a.grad.shape == a.shape and torch.equal(a.grad.reshape(B * T, d), b.grad)


def test_a_masters_gradient_is_the_calls_own():
    say("block norm, parameters in fp32")
    N, d = 200, 136
    g = torch.Generator(device=DEV).manual_seed(6)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV)
    h, y, gx, gn = (normal(N, d).to(torch.bfloat16) for _ in range(4))
    gate, gamma, gamma_y = (normal(d).requires_grad_() for _ in range(3))
    out = tune.block_norm(h, y, gamma, 1e-5, gate=gate, scale=0.5, gamma_y=gamma_y)
    torch.autograd.backward(out, [gx, gn])
    rounded = [t.detach().to(torch.bfloat16) for t in (gamma, gate, gamma_y)]
    _, _, dk, dgy, dg = LL.ll_block_norm_grad(h, y, rounded[0], 1e-5, gx, gn, gate=rounded[1], scale=0.5, gamma_y=rounded[2])
    for p, want in ((gate, dk), (gamma_y, dgy), (gamma, dg)):
        assert torch.equal(p.grad, want)


def test_other_types_are_refused_still():
    say("block norm, parameters in fp16")
    h = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(TypeError, match="gamma"):
        tune.block_norm(h, h, torch.ones((64,), dtype=torch.float16, device=DEV), 1e-5)
