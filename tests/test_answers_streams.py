"""Calls that learn from answers on a stream of their own: copies of batches, results and workspaces are that stream's (no GPU needed)."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests import test_call_streams as T

each = lambda dtype=torch.float32: T.across(T.B, T.T, dtype=dtype)  # noqa: E731
ids = lambda: each(torch.int32)  # noqa: E731
offsets = lambda: torch.zeros((5,), dtype=torch.int32)  # noqa: E731

CALLS = {
    "ll_policy": (6, lambda s: LL.ll_policy(T.across(T.B, T.T, T.d), T.weights(), ids(), each(), each(), ref_logp=each(), weight=each(), stream=s)),
    "ll_preference": (3, lambda s: LL.ll_preference(T.across(T.B, T.T, T.d), T.weights(), ids(), offsets(), ref_logp=each(), stream=s)),
}


@pytest.fixture(autouse=True)
def streams_are_no_objects(request, monkeypatch):
    if "goes" not in request.node.name and "two_devices" not in request.node.name:
        monkeypatch.setattr(LL, "_here", lambda *a: None)


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("given", [True, False])
def test_copies_are_made_on_the_calls_stream(monkeypatch, name, given):
    monkeypatch.setitem(T.CALLS, name, CALLS[name])
    T.test_copies_are_made_on_the_calls_stream(monkeypatch, name, given)


@pytest.mark.parametrize("name", [*CALLS, "ll_grad_norm"])
def test_results_and_workspaces_are_memory_of_the_calls_stream(monkeypatch, name):
    grads = LL.TensorList([])
    call = CALLS[name][1] if name in CALLS else lambda s: LL.ll_grad_norm(grads, stream=s)
    grads.device = torch.device("cpu")
    monkeypatch.setitem(T.MAKES, name, call)
    T.test_results_and_workspaces_are_memory_of_the_calls_stream(monkeypatch, name)


@pytest.mark.parametrize("index,stream,fails", [(0, None, False), (1, None, True), (1, 0, False), (0, 1, True)])
def test_the_call_goes_to_the_device_of_its_tensors(monkeypatch, index, stream, fails):
    """index: the current device; stream: the given one's; the tensors are on device 0."""
    monkeypatch.setattr(LL, "_device", lambda: index)
    given = None if stream is None else type("Stream", (), {"device": torch.device("cuda", stream)})()
    if fails:
        with pytest.raises(ValueError, match="goes to device 1"):
            LL._here(torch.device("cuda:0"), given)
    else:
        LL._here(torch.device("cuda:0"), given)


def test_tensors_on_two_devices():
    with pytest.raises(ValueError, match="cpu and on meta"):
        LL._here(torch.device("cpu"), None, None, torch.zeros(1), torch.zeros(1, device="meta"))
