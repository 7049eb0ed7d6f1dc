"""Training through the lens: the calls under autograd, and a translator that learns."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from paper_2604_06483_amd import tune
from tests.conftest import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_autograd_passes_on_what_the_calls_return():
    say("autograd")
    N, d, V, k = 40, 128, 900, 5
    g = torch.Generator(device=DEV).manual_seed(4)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV).to(torch.bfloat16)
    h, y, gate, gamma, gamma_y, W = normal(N, d), normal(N, d), normal(d), normal(d), normal(d), normal(V, d)
    ids = torch.randint(0, V, (N, k), generator=g, device=DEV, dtype=torch.int32)
    scores = normal(N, k).float()
    leaves = [t.clone().requires_grad_() for t in (h, y, gate, gamma, gamma_y)]
    x, n = tune.block_norm(leaves[0], leaves[1], leaves[3], 1e-5, gate=leaves[2], scale=0.5, gamma_y=leaves[4])
    gx, gn = normal(N, d), normal(N, d)
    torch.autograd.backward([x, n], [gx, gn])
    dh, dy, dk, dgy, dg = LL.ll_block_norm_grad(h, y, gamma, 1e-5, gx, gn, gate=gate, scale=0.5, gamma_y=gamma_y)
    for leaf, want in zip(leaves, (dh, dy, dk, dg, dgy)):
        assert torch.equal(leaf.grad, want.to(torch.bfloat16))
    rows = n.detach().clone().requires_grad_()
    logp, entropy = tune.token_logp(rows, W, ids, temperature=0.5)
    g_logp, g_entropy = torch.randn((N, k), generator=g, device=DEV), torch.randn((N,), generator=g, device=DEV)
    torch.autograd.backward([logp, entropy], [g_logp, g_entropy])
    a, lse, b = LL.ll_logp(rows.detach(), W, ids, temperature=0.5)
    assert torch.equal(logp, a) and torch.equal(entropy, b)
    assert torch.equal(rows.grad, LL.ll_logp_grad(rows.detach(), W, ids, lse, b, g_logp, g_entropy, temperature=0.5))
    rows = n.detach().clone().requires_grad_()
    weight = torch.rand((N,), generator=g, device=DEV)
    loss = tune.distill(rows, W, ids, scores, temperature=2.0, weight=weight)
    loss.sum().backward()
    want, grad = LL.ll_distill(rows.detach(), W, ids, scores, temperature=2.0, weight=weight)
    assert torch.equal(loss, weight * want) and torch.equal(rows.grad, grad)


def test_rows_in_more_than_one_dimension():
    """As the calls take them: the block's output as a matrix beside hidden states with a batch in front."""
    say("autograd, batches")
    B, T, d, V, k = 2, 9, 64, 300, 3
    g = torch.Generator(device=DEV).manual_seed(8)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV).to(torch.bfloat16)
    gamma, W = normal(d), normal(V, d)
    ids = torch.randint(0, V, (B * T, k), generator=g, device=DEV, dtype=torch.int32)
    scores = normal(B * T, k).float()
    h, y = normal(B, T, d).requires_grad_(), normal(B * T, d).requires_grad_()
    flat = [t.detach().reshape(B * T, d).clone().requires_grad_() for t in (h, y)]
    for a, b in ((h, y), flat):
        n = tune.block_norm(a, b, gamma, 1e-5)[1]
        logp, entropy = tune.token_logp(n, W, ids)
        (tune.distill(n, W, ids, scores).sum() + logp.sum() + entropy.sum()).backward()
    assert h.grad.shape == h.shape and y.grad.shape == y.shape
    assert torch.equal(h.grad.reshape(B * T, d), flat[0].grad) and torch.equal(y.grad, flat[1].grad)


def test_a_second_derivative_is_refused():
    """The gradients are the library's, and it has none of theirs: an error, and no silent zeros."""
    say("autograd, twice")
    N, d, V, k = 12, 64, 200, 3
    g = torch.Generator(device=DEV).manual_seed(9)
    rows, y = (torch.randn((N, d), generator=g, device=DEV).to(torch.bfloat16).requires_grad_() for _ in range(2))
    gamma, W = (torch.randn(s, generator=g, device=DEV).to(torch.bfloat16) for s in ((d,), (V, d)))
    ids = torch.randint(0, V, (N, k), generator=g, device=DEV, dtype=torch.int32)
    scores = torch.randn((N, k), generator=g, device=DEV)
    factor = torch.ones((), device=DEV, requires_grad=True)          # so that the gradient depends on something that wants one
    for value in (tune.block_norm(rows, y, gamma, 1e-5)[1].float().sum(), tune.token_logp(rows, W, ids)[0].sum(), tune.distill(rows, W, ids, scores).sum()):
        (grad,) = torch.autograd.grad(factor * value, rows, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            grad.float().sum().backward()


def test_a_translator_learns():
    """The inner rows' raw lens does not know the last layer's token; after some steps it does, and the loss has fallen by half."""
    say("translator")
    inner, last, gamma, W = tune.synthetic_layers(512, 128, 1000, DEV)
    result = tune.fit(tune.Translator(128, gamma, 1e-5), inner, last, W, k=8, steps=150, rate=3e-3)
    assert result.losses[-1] < 0.5 * result.losses[0], result
    assert result.logp_after > result.logp_before + 0.5, result
