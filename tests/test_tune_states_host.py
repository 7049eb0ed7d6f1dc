"""The optimiser's states: replaced one by one, loaded through torch's hooks, and copies that autograd knows of (no GPU needed)."""
import copy

import torch

from paper_2604_06483_amd import tune
from tests.test_tune_answers_host import List, steps  # noqa: F401


def stepped(bits=8):
    a = torch.nn.Parameter(torch.ones(300))
    opt = tune.AdamW([a], bits=bits)
    a.grad = torch.ones(300)
    opt.step()
    return a, opt


def test_a_state_in_other_memory_is_another(steps):  # noqa: F811
    """Any of them: a list that is kept would go on with the old."""
    a, opt = stepped()
    for name in ("m", "v", "m_scale", "v_scale"):
        opt.state[a][name] = opt.state[a][name].clone()
        made = List.made
        opt.step()
        assert List.made == made + 1, name
        opt.step()
        assert List.made == made + 1, name
    opt.state[a]["average"] = torch.ones(300)             # (a program's own beside them)
    opt.step()
    assert List.made == made + 1


def test_a_copied_optimiser_loads(steps):  # noqa: F811
    a, opt = stepped()
    b, other = copy.deepcopy((a, opt))
    other.state[b]["step"] = 7
    other.load_state_dict(opt.state_dict())
    assert other.state[b]["step"] == 1 and other.state[b]["v"].dtype == torch.float8_e5m2


def test_hooks_after_loading_see_the_states_as_they_are(steps):  # noqa: F811
    a, opt = stepped()
    b = torch.nn.Parameter(a.detach().clone())
    other, seen = tune.AdamW([b], bits=8), []
    other.register_load_state_dict_post_hook(lambda o: seen.append({k: x.dtype for k, x in o.state[b].items() if k != "step"}))
    other.load_state_dict(opt.state_dict())
    assert seen == [dict(m=torch.float8_e4m3fn, v=torch.float8_e5m2, m_scale=torch.float32, v_scale=torch.float32)]
    other.load_state_dict(opt.state_dict())
    assert len(seen) == 2


def test_what_a_hook_before_loading_returns_is_loaded(steps):  # noqa: F811
    a, opt = stepped()
    b = torch.nn.Parameter(a.detach().clone())
    other = tune.AdamW([b], bits=8)

    def forgets(o, given):
        state = {i: dict(s, step=40, m=torch.zeros(300, dtype=torch.uint8).view(torch.float8_e4m3fn)) for i, s in given["state"].items()}
        return dict(given, state=state)

    hook = other.register_load_state_dict_pre_hook(forgets)
    other.load_state_dict(opt.state_dict())
    assert other.state[b]["step"] == 40 and not other.state[b]["m"].view(torch.uint8).any() and opt.state[a]["step"] == 1
    hook.remove()
    other.load_state_dict(opt.state_dict())
    assert other.state[b]["step"] == 1 and other.state[b]["m"].view(torch.uint8).any()


def test_autograd_knows_that_a_copy_is_another(steps):  # noqa: F811
    a = torch.nn.Parameter(torch.ones(8))
    mine = a.detach().bfloat16()
    b = torch.nn.Parameter(torch.ones(8))
    opt = tune.AdamW([a, b], copies={a: mine, b: None})
    a.grad = b.grad = torch.ones(8)
    before = mine._version
    opt.step()
    assert mine._version > before
