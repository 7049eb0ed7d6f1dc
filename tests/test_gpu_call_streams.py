"""Calls on a stream of their own, with batches that have to be copied to be rows, while the current stream is busy."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.conftest import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, T, d, V, k = 24, 50, 256, 3000, 4


def inputs():
    g = torch.Generator(device=DEV).manual_seed(7)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV)
    batch = lambda: normal(T, B, d).to(torch.bfloat16).transpose(0, 1)
    t = dict(h=batch(), y=batch(), gx=batch(), gn=batch(), gamma=normal(d).to(torch.bfloat16), W=(0.1 * normal(V, d)).to(torch.bfloat16),
             v=normal(d), ids=torch.randint(0, V, (T, B, k), generator=g, device=DEV, dtype=torch.int32).transpose(0, 1),
             scores=normal(T, B, k).transpose(0, 1), g_logp=normal(T, B, k).transpose(0, 1), g_ent=normal(B * T))
    t["lse"], t["ent"] = LL.ll_logp(t["h"].contiguous(), t["W"], t["ids"].contiguous())[1:]
    return t


CALLS = {
    "project": lambda t, s: LL.ll_project(t["h"], t["gamma"], t["W"], 1e-5, k, stream=s),
    "inject": lambda t, s: LL.ll_steer_inject(t["h"], t["gamma"], 1e-5, t["v"], 0.5, stream=s),
    "inject raw": lambda t, s: LL.ll_steer_inject_raw(t["h"], t["v"], 0.5, stream=s),
    "sweep": lambda t, s: LL.ll_steer_sweep(t["h"], t["gamma"], t["W"], 1e-5, t["v"], [0.0, 1.0], stream=s),
    "block norm": lambda t, s: LL.ll_block_norm(t["h"], t["y"], t["gamma"], 1e-5, stream=s),
    "block norm grad": lambda t, s: LL.ll_block_norm_grad(t["h"], t["y"], t["gamma"], 1e-5, t["gx"], t["gn"], stream=s),
    "logp": lambda t, s: LL.ll_logp(t["h"], t["W"], t["ids"], stream=s),
    "logp grad": lambda t, s: LL.ll_logp_grad(t["h"], t["W"], t["ids"], t["lse"], t["ent"], t["g_logp"], t["g_ent"], stream=s),
    "distill": lambda t, s: LL.ll_distill(t["h"], t["W"], t["ids"], t["scores"], stream=s),
}


@pytest.mark.parametrize("name", CALLS)
def test_batches_are_copied_where_the_call_goes(name):
    say(f"a batch copied on the call's stream: {name}")
    t = inputs()
    call = CALLS[name]
    both = lambda out: [x for x in (out if isinstance(out, tuple) else (out,)) if x is not None]
    want = both(call({n: x.contiguous() for n, x in t.items()}, None))
    side, busy = torch.cuda.Stream(), torch.randn((4096, 4096), device=DEV)
    other = torch.empty_like(busy)
    torch.cuda.synchronize()
    for _ in range(4):                      # some milliseconds on the current stream, which the call does not wait for
        torch.matmul(busy, busy, out=other)
    got = both(call(t, side))
    side.synchronize()
    assert len(got) == len(want)
    for a, b in zip(got, want):
        assert torch.equal(a.reshape(b.shape).nan_to_num(7.0), b.nan_to_num(7.0))
    torch.cuda.synchronize()
