"""What a call on a stream of its own makes, copies of batches that are no rows, results and workspaces, is that stream's (no GPU needed)."""
import contextlib

import pytest
import torch
from torch.overrides import TorchFunctionMode

from paper_2604_06483_amd import binding as LL

B, T, d, V, k = 3, 4, 16, 20, 2
BF16 = torch.bfloat16


class Library:
    """Every call succeeds, every workspace is small."""

    def __getattr__(self, name):
        return lambda *a: 256 if name.endswith("_bytes") else 0


def across(*size, dtype=BF16):
    """[B, T, ...] in the order of a [T, B, ...]: no rows without a copy."""
    return torch.zeros((size[1], size[0], *size[2:]), dtype=dtype).transpose(0, 1)


def vector(dtype=BF16):
    return torch.zeros((d,), dtype=dtype)


def weights():
    return torch.zeros((V, d), dtype=BF16)


def ids():
    return across(B, T, k, dtype=torch.int32)


def scores():
    return across(B, T, k, dtype=torch.float32)


def row():
    return torch.zeros((B * T,))


CALLS = {   # and how many of the inputs are such batches
    "ll_project": (1, lambda s: LL.ll_project(across(B, T, d), vector(), weights(), 1e-5, k, stream=s)),
    "ll_project_static": (1, lambda s: LL.ll_project_static(across(B, T, d), vector(), weights(), 1e-5, k, stream=s)),
    "ll_steer_inject": (1, lambda s: LL.ll_steer_inject(across(B, T, d), vector(), 1e-5, vector(torch.float32), 1.0, stream=s)),
    "ll_steer_inject_raw": (1, lambda s: LL.ll_steer_inject_raw(across(B, T, d), vector(torch.float32), 1.0, stream=s)),
    "ll_steer_sweep": (1, lambda s: LL.ll_steer_sweep(across(B, T, d), vector(), weights(), 1e-5, vector(torch.float32), [1.0], stream=s)),
    "ll_block_norm": (2, lambda s: LL.ll_block_norm(across(B, T, d), across(B, T, d), vector(), 1e-5, stream=s)),
    "ll_block_norm_grad": (4, lambda s: LL.ll_block_norm_grad(*[across(B, T, d) for _ in range(2)], vector(), 1e-5,
                                                              *[across(B, T, d) for _ in range(2)], stream=s)),
    "ll_logp": (2, lambda s: LL.ll_logp(across(B, T, d), weights(), ids(), stream=s)),
    "ll_logp_grad": (3, lambda s: LL.ll_logp_grad(across(B, T, d), weights(), ids(), row(), row(), scores(), stream=s)),
    "ll_distill": (3, lambda s: LL.ll_distill(across(B, T, d), weights(), ids(), scores(), stream=s)),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("given", [True, False])
def test_copies_are_made_on_the_calls_stream(monkeypatch, name, given):
    there, mine, copies = [None], object(), []

    @contextlib.contextmanager
    def on(stream):
        before, there[0] = there[0], stream
        yield
        there[0] = before

    class Copies(TorchFunctionMode):
        def __torch_function__(self, func, types, args=(), kwargs=None):
            out = func(*args, **(kwargs or {}))
            if func is torch.Tensor.reshape and out.data_ptr() != args[0].data_ptr():
                copies.append(there[0])
            return out

    plain = lambda size, dtype, device, stream: torch.empty(size, dtype=dtype)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(LL, "_lib", Library())
    monkeypatch.setattr(LL, "_check", lambda *a, **kw: None)
    monkeypatch.setattr(LL, "_stream", lambda s: 0)
    monkeypatch.setattr(LL, "_scratch", lambda n, device, stream: torch.empty(256, dtype=torch.uint8))
    monkeypatch.setattr(LL, "_empty", plain)
    monkeypatch.setattr(LL, "_like", lambda t, stream: torch.empty_like(t))
    count, call = CALLS[name]
    with Copies():
        call(mine if given else None)
    assert copies == [mine if given else None] * count


MAKES = {n: call for n, (_, call) in CALLS.items()}
MAKES["ll_steer_vector"] = lambda s: LL.ll_steer_vector(weights(), weights(), stream=s)


@pytest.mark.parametrize("name", MAKES)
def test_results_and_workspaces_are_memory_of_the_calls_stream(monkeypatch, name):
    """Memory of the current stream's may still be read by what was queued there before it was freed."""
    there, mine, current, made, kept = [None], object(), object(), [], []

    @contextlib.contextmanager
    def on(stream):
        before, there[0] = there[0], stream
        yield
        there[0] = before

    class Made(TorchFunctionMode):
        def __torch_function__(self, func, types, args=(), kwargs=None):
            if func in (torch.empty, torch.empty_like):
                made.append(there[0])
            return func(*args, **(kwargs or {}))

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept.append(s))
    monkeypatch.setattr(LL, "_lib", Library())
    monkeypatch.setattr(LL, "_check", lambda *a, **kw: None)
    monkeypatch.setattr(LL, "_stream", lambda s: 0)
    with Made():
        MAKES[name](mine)
    assert made and all(s is mine for s in made) and kept == [current] * len(made)


@pytest.mark.parametrize("whole", [True, False])
def test_a_gate_may_have_the_batch_of_its_rows(monkeypatch, whole):
    def shapes(t, dtype, name, shape=None):
        if shape is not None and t.shape != shape:
            raise ValueError(name)
        assert t.is_contiguous(), name

    monkeypatch.setattr(LL, "_lib", Library())
    monkeypatch.setattr(LL, "_check", shapes)
    monkeypatch.setattr(LL, "_stream", lambda s: 0)
    h = torch.zeros((B, T, d), dtype=BF16)
    gate = torch.zeros((B, T, d), dtype=BF16) if whole else across(B, T, d)
    LL.ll_block_norm(h, h, vector(), 1e-5, gate=gate)
    assert LL.ll_block_norm_grad(h, h, vector(), 1e-5, None, h, gate=gate)[2].shape == (B, T, d)
    for wrong in (gate[:, :2], gate[..., :8], gate[0], vector()[:8], torch.zeros((), dtype=BF16)):
        with pytest.raises(ValueError, match="gate"):
            LL.ll_block_norm(h, h, vector(), 1e-5, gate=wrong)
