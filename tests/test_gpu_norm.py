"""ll_block_norm and ll_block_norm_grad against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle.learn_oracle as O
from paper_2604_06483_amd import binding as LL
from tests.conftest import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# A value rounded to bf16 once is off by at most half of the spacing, 2^-7 of the power of two below it, so 2^-8 of itself; fp32
# arithmetic in between by some 2^-24 for each of at most ~100 dependent roundings (the statistics' sums among them) of what it is made of.
BF16 = 2.0 ** -8
FP32 = 100 * 2.0 ** -24

SIZES = [(1, 8), (3, 72), (2, 512), (33, 4096), (5, 4104), (2, 8192), (3, 8200), (2, 16384), (300, 12296), (777, 264), (2500, 64), (1100, 1608)]


def inputs(N, d, gate, post, seed=0):
    g = torch.Generator().manual_seed(100 * N + d + seed)
    normal = lambda *s: torch.randn(s, generator=g)
    outliers = torch.ones(d)
    outliers[torch.randint(0, d, (2,), generator=g)] = 20.0
    t = dict(hidden=3 * normal(N, d) * outliers, y=normal(N, d), gamma=1 + 0.1 * normal(d), g_hidden=normal(N, d), g_normed=normal(N, d),
             gate=None if gate == "none" else 0.5 + 0.3 * normal(*((d,) if gate == "shared" else (N, d))),
             gamma_y=1 + 0.1 * normal(d) if post else None)
    return {n: None if x is None else x.to(torch.bfloat16) for n, x in t.items()}


def f64(x):
    return None if x is None else x.double().cpu().numpy()


def on_gpu(t):
    return {n: None if x is None else x.to(DEV) for n, x in t.items()}


def close(got, ref, size, bits, what):
    got = f64(got)
    bound = (BF16 * np.abs(ref) if bits == 16 else 2.0 ** -24 * np.abs(ref)) + FP32 * size + 1e-37
    bad = np.abs(got - ref) > bound
    assert not bad.any(), (what, int(bad.sum()), float(np.max(np.abs(got - ref) / bound)))


def check(t, eps, scale, N):
    c, r = on_gpu(t), {n: f64(x) for n, x in t.items()}
    opt = dict(gate=c["gate"], scale=scale, gamma_y=c["gamma_y"])
    ref_opt = dict(gate=r["gate"], scale=scale, gamma_y=r["gamma_y"])
    x, n = LL.ll_block_norm(c["hidden"], c["y"], c["gamma"], eps, **opt)
    rx, rn = O.block_norm(r["hidden"], r["y"], r["gamma"], eps, **ref_opt)
    u = r["y"] if r["gamma_y"] is None else np.abs(r["gamma_y"] * r["y"]) / O._rms(r["y"], eps)
    size = np.abs(r["hidden"]) + np.abs(scale * (1 if r["gate"] is None else r["gate"]) * u)
    close(x, rx, size, 16, "x")
    close(n, rn, np.abs(r["gamma"]) * size / O._rms(rx, eps), 16, "normed")

    got = LL.ll_block_norm_grad(c["hidden"], c["y"], c["gamma"], eps, c["g_hidden"], c["g_normed"], **opt)
    g_hidden = np.zeros_like(r["hidden"]) if r["g_hidden"] is None else r["g_hidden"]
    ref, sizes = O.block_norm_grad(r["hidden"], r["y"], r["gamma"], eps, g_hidden, r["g_normed"], **ref_opt)
    sums = 1 + N * 2.0 ** -24 / FP32      # a sum over the rows has a rounding more for each
    for q, name in ((0, "d_hidden"), (1, "d_y")):
        close(got[q], ref[q], sizes[q], 16, name)
    if t["gate"] is None:
        assert got[2] is None
    elif t["gate"].dim() == 1:
        close(got[2], ref[2].sum(0), sums * sizes[2].sum(0), 32, "d_gate")
    else:
        close(got[2], ref[2], sizes[2], 16, "d_gate rows")
    if t["gamma_y"] is None:
        assert got[3] is None
    else:
        close(got[3], ref[3], sums * sizes[3], 32, "d_gamma_y")
    close(got[4], ref[4], sums * sizes[4], 32, "d_gamma")
    return (x, n), got


@pytest.mark.parametrize("N,d", SIZES)
@pytest.mark.parametrize("gate", ["none", "shared", "rows"])
@pytest.mark.parametrize("post", [False, True])
def test_against_the_oracle(N, d, gate, post):
    say(f"block norm N={N} d={d} gate={gate} post={post}")
    check(inputs(N, d, gate, post), 1e-5, 0.5, N)


def test_rows_of_zeros_and_nothing_from_the_stream():
    say("block norm, rows of zeros, no g_hidden")
    t = inputs(9, 264, "rows", True)
    for name in ("hidden", "y"):
        t[name][3] = 0
    t["y"][4] = 0
    t["hidden"][5] = 0
    t["gate"][6] = 0
    t["g_hidden"] = None
    check(t, 1e-5, -1.25, 9)


def test_a_row_that_is_no_number_stays_by_itself():
    say("block norm, NaN and infinity in two rows")
    t = inputs(7, 264, "shared", True)
    clean = check(t, 1e-5, 1.0, 7)
    t["hidden"][2, 5], t["y"][4, 3] = float("nan"), float("inf")
    c = on_gpu(t)
    x, n = LL.ll_block_norm(c["hidden"], c["y"], c["gamma"], 1e-5, gate=c["gate"], gamma_y=c["gamma_y"])
    got = LL.ll_block_norm_grad(c["hidden"], c["y"], c["gamma"], 1e-5, c["g_hidden"], c["g_normed"], gate=c["gate"], gamma_y=c["gamma_y"])
    others = [0, 1, 3, 5, 6]
    for a, b in ((x, clean[0][0]), (n, clean[0][1]), (got[0], clean[1][0]), (got[1], clean[1][1])):
        assert torch.equal(a[others], b[others])
    assert torch.isnan(n[2]).all() and torch.isnan(got[0][2]).all() and torch.isnan(n[4]).any()


@pytest.mark.parametrize("N,d", [(5, 264), (1300, 2560)])
def test_the_same_bits_twice_in_place_and_from_any_workspace(N, d):
    say(f"block norm again, in place N={N} d={d}")
    c = on_gpu(inputs(N, d, "shared", True))
    opt = dict(gate=c["gate"], scale=0.5, gamma_y=c["gamma_y"])
    x, n = LL.ll_block_norm(c["hidden"], c["y"], c["gamma"], 1e-5, **opt)
    hidden, y = c["hidden"].clone(), c["y"].clone()
    LL.ll_block_norm(hidden, y, c["gamma"], 1e-5, out=(hidden, y), **opt)
    assert torch.equal(hidden, x) and torch.equal(y, n)
    need = LL.ll_block_norm_grad_workspace_bytes(N, d)
    results = []
    for fill in (0, 255):
        ws = torch.full((need,), fill, dtype=torch.uint8, device=DEV)
        results.append(LL.ll_block_norm_grad(c["hidden"], c["y"], c["gamma"], 1e-5, c["g_hidden"], c["g_normed"], workspace=ws, **opt))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_no_rows():
    say("block norm of no rows")
    d = 64
    e = torch.empty((0, d), dtype=torch.bfloat16, device=DEV)
    v = torch.ones((d,), dtype=torch.bfloat16, device=DEV)
    x, n = LL.ll_block_norm(e, e, v, 1e-5, gate=v)
    assert x.shape == n.shape == (0, d)
    dh, dy, dk, dgy, dg = LL.ll_block_norm_grad(e, e, v, 1e-5, e, e, gate=v, gamma_y=v)
    assert dh.shape == dy.shape == (0, d) and not dk.any() and not dgy.any() and not dg.any()


def test_on_another_stream_and_in_a_graph():
    say("block norm on a stream of its own, and captured")
    c = on_gpu(inputs(300, 1024, "shared", True))
    opt = dict(gate=c["gate"], scale=0.5, gamma_y=c["gamma_y"])

    def both(stream=None, **more):
        out = LL.ll_block_norm(c["hidden"], c["y"], c["gamma"], 1e-5, stream=stream, **opt)
        return [*out, *LL.ll_block_norm_grad(c["hidden"], c["y"], c["gamma"], 1e-5, c["g_hidden"], c["g_normed"], stream=stream, **opt, **more)]

    eager = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = both(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(eager, there):
        assert torch.equal(a, b)
    ws = torch.empty((LL.ll_block_norm_grad_workspace_bytes(300, 1024),), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both(workspace=ws)
    for turn in range(3):
        for t in captured:
            t.zero_()
        c["hidden"].copy_(c["hidden"].flip(0))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, both()):
            assert torch.equal(a, b), turn


@pytest.mark.parametrize("N,d", [(270000, 8192), ((1 << 21) + 3, 64)])
def test_offsets_past_32_bits_and_rows_past_a_launch(N, d):
    """The last rows of a long call are those of a call of them alone."""
    say(f"block norm N={N} d={d}")
    g = torch.Generator(device=DEV).manual_seed(3)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.bfloat16)
    h, y, k, gn, gamma = normal(N, d), normal(N, d), normal(N, d), normal(N, d), normal(d)
    x, n = LL.ll_block_norm(h, y, gamma, 1e-5, gate=k)
    dh, dy, dk, _, _ = LL.ll_block_norm_grad(h, y, gamma, 1e-5, None, gn, gate=k)
    last = slice(N - 5, N)
    part = [t[last].contiguous() for t in (h, y, k, gn)]
    x2, n2 = LL.ll_block_norm(part[0], part[1], gamma, 1e-5, gate=part[2])
    dh2, dy2, dk2, _, _ = LL.ll_block_norm_grad(part[0], part[1], gamma, 1e-5, None, part[3], gate=part[2])
    for a, b in ((x, x2), (n, n2), (dh, dh2), (dy, dy2), (dk, dk2)):
        assert torch.equal(a[last], b)
