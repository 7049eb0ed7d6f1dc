"""ll_block_norm_grad where a workgroup has several wide rows, and written over its own inputs."""
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from tests.conftest import say
from tests.test_gpu_norm import check, inputs, on_gpu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("d", [4104, 8192, 8200, 16384])
@pytest.mark.parametrize("gate", ["none", "shared", "rows"])
@pytest.mark.parametrize("post", [False, True])
def test_sums_over_a_workgroups_rows(d, gate, post):
    """One workgroup a compute unit at these widths, so that most have four rows and some five: sums for the parameters carried over them, the next
    row loaded ahead, places of the reductions used again."""
    N = 1100
    say(f"several wide rows a workgroup d={d} gate={gate} post={post}")
    groups = LL.ll_block_norm_grad_workspace_bytes(N, d) // (3 * 4 * d)
    assert N / groups > 4
    check(inputs(N, d, gate, post), 1e-5, 0.5, N)


def raw_grad(c, dh, dy, dk, scale):
    N, d = c["hidden"].shape
    rows = c["gate"] is not None and c["gate"].dim() == 2
    sums = [torch.empty((d,), device=DEV) for _ in range(2)]
    need = LL.ll_block_norm_grad_workspace_bytes(N, d)
    ws = torch.empty((need,), dtype=torch.uint8, device=DEV)
    p = LL._ptr
    rc = LL.lib().ll_block_norm_grad(LL.ll_shape(N, d, 0), p(ws), need, p(c["hidden"]), p(c["y"]), p(c["gate"]), int(rows), scale, p(c["gamma_y"]), p(c["gamma"]),
                                     1e-5, p(c["g_hidden"]), p(c["g_normed"]), p(dh), p(dy), p(dk), p(sums[0]) if c["gamma_y"] is not None else None,
                                     p(sums[1]), LL._stream(None))
    assert rc == LL.LL_OK
    return sums[:1] * (c["gamma_y"] is not None) + sums[1:]


@pytest.mark.parametrize("N,d", [(700, 264), (700, 8192), (700, 12296)])
@pytest.mark.parametrize("gate,post", [("none", False), ("shared", False), ("shared", True), ("rows", True)])
@pytest.mark.parametrize("over", [("hidden", "y"), ("y", "hidden"), ("g_hidden", "g_normed"), ("g_normed", "g_hidden"), ("gate", "hidden"), ("g_hidden", "gate")])
def test_gradients_written_over_the_inputs(N, d, gate, post, over):
    """d_hidden and d_y may be any two [N, d] inputs' own buffers."""
    if "gate" in over and gate != "rows":
        over = tuple("y" if n == "gate" else n for n in over)
    say(f"block norm gradient over its inputs N={N} d={d} gate={gate} post={post} {over}")
    c = on_gpu(inputs(N, d, gate, post))
    like = lambda: torch.empty((N, d), dtype=torch.bfloat16, device=DEV)
    dk = None if gate == "none" else like() if gate == "rows" else torch.empty((d,), device=DEV)
    dh, dy = like(), like()
    sums = raw_grad(c, dh, dy, dk, 0.5)
    again = {n: None if x is None else x.clone() for n, x in c.items()}
    dk2 = None if dk is None else torch.empty_like(dk)
    sums2 = raw_grad(again, again[over[0]], again[over[1]], dk2, 0.5)
    assert torch.equal(again[over[0]], dh) and torch.equal(again[over[1]], dy) and (dk is None or torch.equal(dk2, dk))
    for a, b in zip(sums, sums2):
        assert torch.equal(a, b)
