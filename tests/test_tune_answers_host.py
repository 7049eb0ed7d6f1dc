"""What autograd is told of the calls that learn from answers, and the optimiser's book-keeping, with the calls themselves in torch (no GPU needed)."""
import copy

import pytest
import torch

from paper_2604_06483_amd import tune

N, d, V = 7, 8, 12
OFFSETS = torch.tensor([0, 2, 2, 3, 6], dtype=torch.int32)     # the second sequence is empty, row 6 is in none


def token_logp(rows, W_U, ids, temperature):
    return torch.log_softmax(rows @ W_U.detach().float().t() / temperature, 1).gather(1, ids.long()[:, None])[:, 0]


def plain_policy(rows, W_U, ids, advantage, old_logp=None, *, ref_logp=None, weight=None, clip=(0.2, 0.2), kl=0.0, temperature=1.0, grad=True):
    with torch.enable_grad():
        a = rows.detach().float().reshape(-1, d).requires_grad_()
        logp = token_logp(a, W_U, ids.reshape(-1), temperature)
        loss = -torch.exp(logp - (logp.detach() if old_logp is None else old_logp)) * advantage.reshape(-1)
        out = torch.autograd.grad((loss if weight is None else weight.detach().reshape(-1) * loss).sum(), a)[0] if grad else None
    return loss.detach(), logp.detach(), None if out is None else out.to(rows.dtype).reshape(rows.shape)


def plain_preference(rows, W_U, ids, offsets, *, ref_logp=None, weight=None, beta=0.1, smoothing=0.0, form="logistic", mean=False, temperature=1.0,
                     grad=True):
    with torch.enable_grad():
        a = rows.detach().float().requires_grad_()
        logp = token_logp(a, W_U, ids, temperature)
        sums = torch.stack([logp[offsets[i]:offsets[i + 1]].sum() for i in range(len(offsets) - 1)]).reshape(-1, 2)
        loss = -torch.nn.functional.logsigmoid(beta * (sums[:, 0] - sums[:, 1]))
        out = torch.autograd.grad((loss if weight is None else weight.detach() * loss).sum(), a)[0].to(rows.dtype) if grad else None
    return loss.detach(), sums.detach(), logp.detach(), out


@pytest.fixture(autouse=True)
def calls(monkeypatch):
    monkeypatch.setattr(tune.LL, "ll_policy", plain_policy)
    monkeypatch.setattr(tune.LL, "ll_preference", plain_preference)


def inputs():
    g = torch.Generator().manual_seed(3)
    rows, W = torch.randn((N, d), generator=g), torch.randn((V, d), generator=g)
    return rows, W, torch.randint(0, V, (N,), generator=g, dtype=torch.int32), torch.randn((N,), generator=g), torch.rand((N,), generator=g)


@pytest.mark.parametrize("trained", [True, False])
@pytest.mark.parametrize("size", [(N,), (1, N)])
def test_policy(trained, size):
    """The weight's gradient is what the row's loss is without it; factors of a loss are factors of its row."""
    rows, W, ids, A, weight = inputs()
    rows, ids, A, weight = rows.reshape(*size, d).requires_grad_(trained), ids.reshape(size), A.reshape(size), weight.reshape(size).requires_grad_()
    factor = torch.arange(1.0, N + 1)
    loss, logp = tune.policy(rows, W, ids, A, weight=weight)
    assert not logp.requires_grad
    (factor * loss).sum().backward()
    want, _, grad = plain_policy(rows, W, ids, A, weight=weight)
    assert torch.equal(weight.grad, (factor * want).reshape(size))
    assert torch.equal(rows.grad, factor.reshape(*size, 1) * grad) if trained else rows.grad is None


@pytest.mark.parametrize("trained", [True, False])
def test_preference(trained):
    """Factors of a pair's loss are factors of its rows, of which one is in no pair."""
    rows, W, ids, _, _ = inputs()
    weight = torch.tensor([0.7, 1.3], requires_grad=True)
    rows.requires_grad_(trained)
    loss, score, logp = tune.preference(rows, W, ids, OFFSETS, weight=weight)
    assert not score.requires_grad and not logp.requires_grad
    factor = torch.tensor([2.0, -3.0])
    (factor * loss).sum().backward()
    want, _, _, grad = plain_preference(rows, W, ids, OFFSETS, weight=weight)
    assert torch.equal(weight.grad, factor * want)
    by = torch.tensor([2.0, 2.0, -3.0, -3.0, -3.0, -3.0, 0.0])
    assert torch.equal(rows.grad, by[:, None] * grad) if trained else rows.grad is None


def test_a_weight_of_zero_passes_nothing_on(monkeypatch):
    rows, W, ids, A, weight = inputs()
    weight[2] = 0.0
    nan = lambda x: torch.where(torch.arange(len(x)) == 2, float("nan"), x)  # noqa: E731
    monkeypatch.setattr(tune.LL, "ll_policy", lambda *a, **k: (nan(torch.ones(N)), torch.ones(N), torch.zeros((N, d))))
    loss, _ = tune.policy(rows.requires_grad_(), W, ids, A, weight=weight)
    assert torch.equal(loss, weight)


def test_what_gets_no_gradient_must_not_ask_for_one():
    rows, W, ids, A, _ = inputs()
    other = torch.zeros((N,))
    uses = {"W_U": lambda: (tune.policy(rows, W, ids, A), tune.preference(rows, W, ids, OFFSETS)), "advantage": lambda: tune.policy(rows, W, ids, A),
            "old_logp": lambda: tune.policy(rows, W, ids, A, other), "ref_logp": lambda: tune.preference(rows, W, ids, OFFSETS, ref_logp=other)}
    for name, use in uses.items():
        wants = {"W_U": W, "advantage": A}.get(name, other).requires_grad_()
        with pytest.raises(ValueError, match=name):
            use()
        with torch.no_grad():
            use()
        wants.requires_grad_(False)
        use()


class List:
    """A TensorList that holds any tensors."""
    made = 0

    def __init__(self, grads, params=None, m=None, v=None, m_scale=None, v_scale=None, copies=None):
        List.made += 1
        kept = lambda of: None if of is None else [None if x is None else x.detach() for x in of]  # noqa: E731
        self.grads, self.params, self.m, self.v, self.copies = kept(grads), kept(params), kept(m), kept(v), kept(copies)

    def set_grads(self, grads):
        self.grads = list(grads)

    def __len__(self):
        return len(self.grads)


@pytest.fixture
def steps(monkeypatch):
    """Plain descent in place of the step; what was called with."""
    seen = []

    def adamw(tensors, step, **kw):
        seen.append((step, len(tensors), kw))
        for i, (p, g) in enumerate(zip(tensors.params, tensors.grads)):
            p.data.sub_(kw["rate"] * g.to(p.dtype))
            tensors.m[i].copy_((tensors.m[i].float() + 1).to(tensors.m[i].dtype))

    monkeypatch.setattr(tune.LL, "TensorList", List)
    monkeypatch.setattr(tune.LL, "ll_adamw", adamw)
    monkeypatch.setattr(tune.LL, "ll_grad_norm", lambda tensors: torch.stack([g.square().sum() for g in tensors.grads]).sum().sqrt().reshape(1))
    List.made = 0
    return seen


def test_a_group_is_one_call_and_its_list_is_kept(steps):
    a, b, c = (torch.nn.Parameter(torch.ones(n)) for n in (3, 300, 5))
    opt = tune.AdamW([{"params": [a, b]}, {"params": [c], "lr": 0.5}], lr=0.1, max_norm=2.0)
    for t in range(3):
        opt.zero_grad(set_to_none=True)
        (a.sum() + b.sum() + c.sum()).backward()
        before = a._version
        opt.step()
        assert a._version > before                        # autograd knows that the parameter is another
    assert [(s, n, kw["rate"]) for s, n, kw in steps] == [(1, 2, 0.1), (1, 1, 0.5), (2, 2, 0.1), (2, 1, 0.5), (3, 2, 0.1), (3, 1, 0.5)]
    assert all(float(kw["norm"]) == pytest.approx(308 ** 0.5) and kw["max_norm"] == 2.0 for _, _, kw in steps)
    assert List.made == 2 + 3                             # two groups' once, and the norm's of both
    assert float(opt.norm) == pytest.approx(308 ** 0.5)


def test_parameters_without_a_gradient_count_their_own_steps(steps):
    a, b = torch.nn.Parameter(torch.ones(3)), torch.nn.Parameter(torch.ones(3))
    opt = tune.AdamW([a, b], bits=8)
    a.sum().backward()
    opt.step()
    opt.step()
    b.sum().backward()
    opt.step()
    assert [(s, n) for s, n, _ in steps] == [(1, 1), (2, 1), (3, 1), (1, 1)]
    assert opt.state[a]["m"].dtype == torch.float8_e4m3fn and opt.state[a]["v"].dtype == torch.float8_e5m2 and opt.state[a]["m_scale"].shape == (1,)


@pytest.mark.parametrize("bits,dtype", [(8, torch.float32), (32, torch.bfloat16)])
def test_states_survive_being_saved(steps, bits, dtype):
    """In their own types, and not in the parameter's."""
    a = torch.nn.Parameter(torch.ones(300, dtype=dtype))
    opt = tune.AdamW([a], bits=bits)
    a.sum().backward()
    opt.step()
    b = torch.nn.Parameter(a.detach().clone())
    other = tune.AdamW([b], bits=bits)
    other.load_state_dict(opt.state_dict())
    for k, x in opt.state[a].items():
        y = other.state[b][k]
        assert x == y if k == "step" else x is not y and x.dtype == y.dtype and torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k
    b.grad = a.grad
    other.step()
    assert [s for s, _, _ in steps] == [1, 2]


def test_memory_that_a_parameter_no_longer_has_is_not_stepped(steps):
    a = torch.nn.Parameter(torch.ones(3))
    opt = tune.AdamW([a], lr=0.5)
    a.grad = torch.ones(3)
    opt.step()
    old = a.data
    a.data = torch.full((3,), 7.0)                        # (as moving a model does)
    opt.step()
    assert torch.equal(a.detach(), torch.full((3,), 6.5)) and torch.equal(old, torch.full((3,), 0.5)) and List.made == 2


def test_a_copied_optimiser_goes_on(steps):
    a = torch.nn.Parameter(torch.ones(3))
    opt = tune.AdamW([a], lr=0.5, bits=8, max_norm=2.0, seed=4)
    a.grad = torch.ones(3)
    opt.step()
    b, other = copy.deepcopy((a, opt))
    b.grad = torch.ones(3)
    other.step()
    assert [s for s, _, _ in steps] == [1, 2] and steps[1][2]["max_norm"] == 2.0 and steps[1][2]["seed"] == 4
    assert torch.equal(b.detach(), torch.zeros(3)) and torch.equal(a.detach(), torch.full((3,), 0.5))


def test_gradients_that_are_no_whole_rows(steps, monkeypatch):
    """Transposed, and from the middle of a buffer: a copy; sparse: an error."""
    a, b = torch.nn.Parameter(torch.zeros(3, 2)), torch.nn.Parameter(torch.zeros(5))
    a.grad, b.grad = torch.arange(6.0).reshape(2, 3).T, torch.arange(9.0)[1:6]
    opt = tune.AdamW([a, b], lr=1.0)
    opt.step()
    assert torch.equal(a.detach(), -a.grad) and torch.equal(b.detach(), -b.grad)
    a.grad = torch.zeros(3, 2).to_sparse()
    with pytest.raises(ValueError, match="dense"):
        opt.step()


def test_refusals():
    a = torch.nn.Parameter(torch.ones(3))
    for bad in (dict(bits=16), dict(max_norm=0.0), dict(max_norm=float("nan"))):
        with pytest.raises(ValueError):
            tune.AdamW([a], **bad)
