"""Memory of a training step with the library's optimiser."""
import gc

import pytest
import torch

from paper_2604_06483_amd import tune
from tests.conftest import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("max_norm", [None, 1.0])
def test_gradients_are_freed_after_a_step(bits, max_norm):
    """Between two steps there are parameters and states."""
    say(f"memory after a step, {bits} bits, max_norm {max_norm}")
    gc.collect()
    n = 1 << 20
    a, b = (torch.nn.Parameter(torch.ones((n,), device=DEV)) for _ in range(2))
    opt = tune.AdamW([{"params": [a]}, {"params": [b], "lr": 0.1}], bits=bits, max_norm=max_norm)
    used = []
    for t in range(3):
        a.grad, b.grad = torch.full((n,), 1.0 + t, device=DEV), torch.zeros((2, n // 2), device=DEV).T.reshape(-1)
        opt.step()
        opt.zero_grad(set_to_none=True)
        used.append(torch.cuda.memory_allocated())
    states = 4 * n if bits == 8 else 16 * n
    scales = 0 if bits == 32 else 4 * 4 * n // 256
    small = 4096                                                  # the norm
    assert used[0] == used[1] == used[2]
    del opt
    assert abs(used[0] - torch.cuda.memory_allocated() - states - scales) <= small
