"""What autograd is told of the calls that learn through the lens, with the calls themselves in torch (no GPU needed)."""
import pytest
import torch

from paper_2604_06483_amd import tune

N, d, V, k = 6, 8, 12, 3


def plain_distill(rows, W_U, teacher_ids, teacher_scores, *, temperature=1.0, weight=None, grad=True):
    with torch.enable_grad():
        a = rows.detach().float().requires_grad_()
        logp = torch.log_softmax(a @ W_U.detach().float().t() / temperature, 1)
        log_t = torch.log_softmax(teacher_scores.detach() / temperature, 1)
        loss = temperature ** 2 * (log_t.exp() * (log_t - logp.gather(1, teacher_ids.long()))).sum(1)
        out = torch.autograd.grad((loss if weight is None else weight.detach() * loss).sum(), a)[0].to(rows.dtype) if grad else None
    return loss.detach(), out


@pytest.fixture
def calls(monkeypatch):
    monkeypatch.setattr(tune.LL, "ll_distill", plain_distill)


def inputs():
    g = torch.Generator().manual_seed(3)
    rows, W = (torch.randn(s, generator=g).to(torch.bfloat16) for s in ((N, d), (V, d)))
    return rows, W, torch.randint(0, V, (N, k), generator=g, dtype=torch.int32), torch.randn((N, k), generator=g), torch.rand((N,), generator=g)


@pytest.mark.parametrize("trained", [True, False])
def test_the_weight_of_a_distillation_gets_its_gradient(calls, trained):
    """It is what the row's loss is without it, whether or not the rows are trained as well."""
    rows, W, ids, scores, weight = inputs()
    rows.requires_grad_(trained)
    weight.requires_grad_()
    factor = torch.arange(1.0, N + 1)
    (factor * tune.distill(rows, W, ids, scores, weight=weight)).sum().backward()
    loss, grad = plain_distill(rows, W, ids, scores, weight=weight)
    assert torch.equal(weight.grad, factor * loss)
    assert torch.equal(rows.grad, (factor[:, None] * grad).to(torch.bfloat16)) if trained else rows.grad is None


def plain_logp(rows, W_U, ids, *, temperature=1.0):
    logp = torch.log_softmax(rows.detach().float() @ W_U.detach().float().t() / temperature, 1)
    return logp.gather(1, ids.long()), torch.zeros((N,)), -(logp.exp() * logp).sum(1)


@pytest.mark.parametrize("which", ["W_U", "teacher_scores"])
def test_what_gets_no_gradient_must_not_ask_for_one(calls, monkeypatch, which):
    """An error, and no training step that misses a term."""
    monkeypatch.setattr(tune.LL, "ll_logp", plain_logp)
    rows, W, ids, scores, _ = inputs()
    rows.requires_grad_()
    wants = {"W_U": W, "teacher_scores": scores}[which].requires_grad_()
    uses = [lambda: tune.distill(rows, W, ids, scores)] + ([lambda: tune.token_logp(rows, W, ids)] if which == "W_U" else [])
    for use in uses:
        with pytest.raises(ValueError, match=which):
            use()
        with torch.no_grad():
            use()                               # read, not trained
    wants.requires_grad_(False)
    for use in uses:
        use()


def test_a_row_of_weight_zero_adds_nothing_whatever_it_holds(monkeypatch):
    loss, grad = torch.tensor([0.5, float("nan"), float("inf"), 2.0]), torch.zeros((4, d), dtype=torch.bfloat16)
    monkeypatch.setattr(tune.LL, "ll_distill", lambda *a, **kw: (loss, grad))
    weight = torch.tensor([0.25, 0.0, -0.0, 0.0], requires_grad=True)
    out = tune.distill(torch.zeros((4, d), dtype=torch.bfloat16), torch.zeros((V, d), dtype=torch.bfloat16), torch.zeros((4, 1), dtype=torch.int32), torch.zeros((4, 1)), weight=weight)
    assert torch.equal(out.detach(), torch.tensor([0.125, 0.0, 0.0, 0.0]))
    out.sum().backward()
    assert torch.equal(weight.grad.nan_to_num(7.0), loss.nan_to_num(7.0))     # (the weight's own gradient is what the row's loss is)


@pytest.fixture
def wide_default():
    before = torch.get_default_dtype()
    torch.set_default_dtype(torch.float64)
    yield
    torch.set_default_dtype(before)


def test_types_do_not_follow_torchs_default(wide_default, monkeypatch):
    """The calls take fp32: what autograd and the translator make themselves is fp32 under any default."""
    seen = []
    monkeypatch.setattr(tune.LL, "ll_logp", lambda rows, W, ids, **kw: tuple(torch.zeros(s, dtype=torch.float32) for s in ((N, k), (N,), (N,))))
    monkeypatch.setattr(tune.LL, "ll_logp_grad", lambda rows, W, ids, lse, ent, g, ge, **kw: seen.append(g.dtype) or torch.zeros_like(rows))
    rows, W, ids, _, _ = inputs()
    rows.requires_grad_()
    tune.token_logp(rows, W, ids)[1].sum().backward()
    assert seen == [torch.float32]
    t = tune.Translator(d, torch.ones((d,), dtype=torch.bfloat16), 1e-5)
    assert {p.dtype for p in t.parameters()} == {torch.float32}


def test_parameters_in_fp32_get_their_sums_unrounded(monkeypatch):
    """gamma, gamma_y and the gate go into the calls as bf16; a master in fp32 gets the fp32 sums over the rows as the call returns them."""
    g = torch.Generator().manual_seed(1)
    sums = [torch.randn((d,), generator=g) for _ in range(3)]
    given = []

    def forward(hidden, y, gamma, eps, *, gate, scale, gamma_y):
        given.extend([gamma, gate, gamma_y])
        return torch.zeros_like(hidden), torch.zeros_like(hidden)

    def backward(hidden, y, gamma, eps, g_hidden, g_normed, *, gate, scale, gamma_y):
        given.extend([gamma, gate, gamma_y])
        return torch.zeros_like(hidden), torch.zeros_like(y), sums[0], sums[1], sums[2]

    monkeypatch.setattr(tune.LL, "ll_block_norm", forward)
    monkeypatch.setattr(tune.LL, "ll_block_norm_grad", backward)
    h = torch.zeros((N, d), dtype=torch.bfloat16)
    for dtype in (torch.float32, torch.bfloat16):
        gate, gamma_y, gamma = (torch.randn((d,), generator=g).to(dtype).requires_grad_() for _ in range(3))
        del given[:]
        tune.block_norm(h, h, gamma, 1e-5, gate=gate, gamma_y=gamma_y)[1].sum().backward()
        for got, p in zip(given, 2 * [gamma, gate, gamma_y]):
            assert got.dtype == torch.bfloat16 and torch.equal(got, p.detach().to(torch.bfloat16))
        for p, s in zip((gate, gamma_y, gamma), sums):
            assert p.grad.dtype == dtype and torch.equal(p.grad, s.to(dtype))
    translator = tune.Translator(d, torch.ones((d,), dtype=torch.bfloat16), 1e-5)
    translator(h).sum().backward()
    assert torch.equal(translator.gate.grad, sums[0])
