"""What the optimiser holds between two steps, and whom it tells, with the calls themselves in torch (no GPU needed)."""
import gc
import weakref

import pytest
import torch

from paper_2604_06483_amd import binding as LL
from paper_2604_06483_amd import tune
from tests.test_tune_answers_host import List, steps  # noqa: F401


def test_gradients_end_with_their_step(steps):  # noqa: F811
    """A gradient that its parameter lets go after a step is nobody's: the next backward pass would have both in memory."""
    a, b = torch.nn.Parameter(torch.ones(300)), torch.nn.Parameter(torch.ones(3, 2))
    opt = tune.AdamW([{"params": [a]}, {"params": [b]}], max_norm=1.0)
    for t in range(3):
        a.grad, b.grad = torch.ones(300), torch.ones(2, 3).T           # (the second is copied)
        held = [weakref.ref(p.grad) for p in (a, b)]
        opt.step()
        opt.zero_grad(set_to_none=True)
        gc.collect()
        assert [r() for r in held] == [None, None], t
        assert all(g is None for kept in lists(opt) for g in kept.grads), t
    assert [s for s, _, _ in steps] == [1, 1, 2, 2, 3, 3]


def lists(opt):
    return [x for kept in opt._lists.values() for x in (kept if isinstance(kept, tuple) else (kept,)) if isinstance(x, List)]


def test_lists_that_a_step_does_not_use_go(steps):  # noqa: F811
    """Parameters that are at different steps have a list each; at one step again they have one, and what nothing uses keeps no memory."""
    a, b, c = (torch.nn.Parameter(torch.ones(3)) for _ in range(3))
    opt = tune.AdamW([{"params": [a, b]}, {"params": [c]}])
    a.grad = c.grad = torch.ones(3)
    opt.step()
    b.grad = torch.ones(3)
    opt.step()
    assert [len(x) for x in lists(opt)] == [1, 1, 1]
    a.grad = None
    opt.step()                                            # b has done as many as a
    a.grad, c.grad = torch.ones(3), None
    opt.step()
    assert sorted(len(x) for x in lists(opt)) == [1, 2]   # (c's is kept for when it has one again)
    made, c.grad = List.made, torch.ones(3)
    opt.step()
    assert List.made == made and [s for s, _, _ in steps] == [1, 1, 2, 1, 2, 2, 3, 3, 4, 4]


def test_a_step_that_fails_holds_no_gradients(steps, monkeypatch):  # noqa: F811
    a = torch.nn.Parameter(torch.ones(300))
    opt = tune.AdamW([a])
    a.grad = torch.ones(300)

    def fails(*args, **kw):
        raise LL.LLError(LL.LL_EHIP, "ll_adamw")

    monkeypatch.setattr(tune.LL, "ll_adamw", fails)
    with pytest.raises(LL.LLError):
        opt.step()
    assert lists(opt) and all(g is None for kept in lists(opt) for g in kept.grads)


def test_a_gradient_that_is_refused_leaves_none_of_the_others(steps):  # noqa: F811
    a, b = (torch.nn.Parameter(torch.ones(4)) for _ in range(2))
    opt = tune.AdamW([{"params": [a]}, {"params": [b]}])
    a.grad = b.grad = torch.ones(4)
    opt.step()
    b.grad = torch.ones(4).to_sparse()
    with pytest.raises(ValueError, match="dense"):
        opt.step()
    assert lists(opt) and all(g is None for kept in lists(opt) for g in kept.grads)


@pytest.fixture
def on_the_cpu(monkeypatch):
    monkeypatch.setattr(LL, "_check", lambda t, dtype, name, shape=None: None if t.dtype == dtype else pytest.fail(name))


def test_a_list_lets_its_gradients_go(on_the_cpu):
    """None in a gradient's place; the call is then refused, and another of the same shape and of either type takes it."""
    x = lambda *s: torch.zeros(s)  # noqa: E731
    many = LL.TensorList([x(8), x(3, 4)], [x(8), x(3, 4)], [x(8), x(3, 4)], [x(8), x(3, 4)])
    flags = [t.flags for t in many.array]
    many.set_grads([None, None])
    assert many.grads == [None, None] and [t.grad for t in many.array] == [None, None]
    assert LL.lib().ll_adamw(many.address, 2, many.options_address, None, None, None, None) == LL.LL_EINVAL
    with pytest.raises(ValueError, match=r"grads\[1\]: shape \(4, 3\)"):
        many.set_grads([x(8), x(4, 3)])
    other = [x(8), x(3, 4).bfloat16()]
    many.set_grads(other)
    assert [t.grad for t in many.array] == [g.data_ptr() for g in other]
    assert [t.flags for t in many.array] == [flags[0], flags[1] | LL.LL_TENSOR_GRAD_BF16]
