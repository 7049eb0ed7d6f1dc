"""The optimiser's states: replaced one by one, loaded through torch's hooks, and copies that autograd knows of (no GPU needed)."""
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
