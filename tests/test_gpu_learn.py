"""ll_logp, ll_logp_grad and ll_distill against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle.learn_oracle as O
from paper_2604_06483_amd import binding as LL
from tests.conftest import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INT_MIN, INT_MAX = -2 ** 31, 2 ** 31 - 1

# (N, d, V, k): one of everything, less than a tile of it, ragged in each direction, more rows than a pass, more ids than a lane has; up
# to eight rows of every width that they are dealt by; the gradient's product in one slice
SIZES = [(1, 8, 1, 1), (1, 64, 5, 2), (3, 72, 257, 3), (64, 256, 4096, 5), (130, 328, 1000, 20), (257, 128, 3001, 64), (300, 1608, 2050, 7),
         (2100, 64, 777, 2), (520, 264, 300, 32), (1, 4096, 33000, 10), (33, 2560, 20000, 10), (17, 200, 70000, 4), (16, 8192, 1500, 1),
         (2, 1000, 3000, 5), (4, 1024, 900, 8), (5, 2048, 700, 3), (8, 4096, 600, 64), (4, 8192, 1000, 4), (3, 5120, 2000, 7), (2, 16384, 500, 2),
         (6, 512, 9000, 10), (7, 2504, 5001, 6), (8, 4104, 300, 3), (3, 8200, 400, 2), (1, 16392, 300, 3), (2, 8, 70000, 33),
         (20, 72, 60, 3), (600, 520, 60, 5), (2048, 8192, 300, 2)]


def inputs(N, d, V, k, spread=8.0, seed=0):
    """Rows near a few tokens' directions: probabilities from 1e-6 to nearly one."""
    g = torch.Generator().manual_seed(1000 * N + d + V + seed)
    W = (0.02 * torch.randn((V, d), generator=g)).to(torch.bfloat16)
    near = torch.randint(0, V, (N, 2), generator=g)
    a = torch.randn((N, d), generator=g)
    for i in range(2):
        a += spread * torch.rand((N, 1), generator=g) / (0.0004 * d) * W[near[:, i]].float()
    a = (a / a.pow(2).mean(1, keepdim=True).sqrt()).to(torch.bfloat16)
    ids = torch.randint(0, V, (N, k), generator=g)
    ids[:, 0] = near[:, 0]
    if k > 3:
        ids[:, 3] = ids[:, 0]                       # a token listed twice
        ids[::2, 2] = -1                            # entries that are none
        ids[1::3, 1] = torch.tensor([V, INT_MIN, INT_MAX])[torch.randint(0, 3, ids[1::3, 1].shape, generator=g)]
    return a, W, ids.to(torch.int32), g


def f64(x):
    return None if x is None else x.double().cpu().numpy()


def logit_error(rows, W, temperature):
    """fp32 sums of products whose sizes add up to at most |a| |w|: a random walk of 2^-24 of that a step of 32 products, in 256 steps
    at most 16 of them; and the exponentials' and logarithms' own last bits, of numbers below 64 in powers of two."""
    n = lambda x: float(np.sqrt(np.max(np.sum(x * x, axis=1))))
    return 16 * 2.0 ** -24 * n(rows) * n(W) / temperature + 4e-6


def grad_close(got, dz, size, W, ez, what):
    """dz is rounded to bf16 at most twice, by up to 2^-8 of itself, rms 2^-8 / sqrt 3 of the power of two below it (0.59 2^-8 of itself
    for both in the mean, 0.82 at most), independently: 4 2^-8 over the root of the squares is six to seven of that.  The result once."""
    ref, got = dz @ W, f64(got)
    bound = 2.0 ** -8 * np.abs(ref) + 8 * 2.0 ** -9 * np.sqrt((dz * dz) @ (W * W)) + 3 * ez * (size @ np.abs(W)) + 1e-37
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(np.abs(got - ref) / bound)))


def check_logp(a, W, ids, g, temperature, entropy=True):
    N, k = ids.shape
    V = W.shape[0]
    r, w = f64(a), f64(W)
    ez = logit_error(r, w, temperature)
    ca, cW, cids = a.to(DEV), W.to(DEV), ids.to(DEV)
    lp, lse, ent = LL.ll_logp(ca, cW, cids, temperature=temperature)
    ref = O.logp(r, w, ids.numpy(), temperature)
    assert np.array_equal(np.isnan(f64(lp)), np.isnan(ref[0]))
    np.testing.assert_allclose(f64(lp), ref[0], rtol=0, atol=2 * ez)
    np.testing.assert_allclose(f64(lse), ref[1], rtol=0, atol=ez + 2.0 ** -23 * float(np.max(np.abs(ref[1]))))
    np.testing.assert_allclose(f64(ent), ref[2], rtol=0, atol=(2 + np.log(V + 1)) * ez)
    g_logp = torch.randn((N, k), generator=g)
    g_ent = torch.randn((N,), generator=g) if entropy else None
    out = LL.ll_logp_grad(ca, cW, cids, lse, ent if entropy else None, g_logp.to(DEV), None if g_ent is None else g_ent.to(DEV),
                          temperature=temperature)
    dz, size = O.logp_grad(r, w, ids.numpy(), f64(g_logp), f64(g_ent), temperature)
    grad_close(out, dz, size, w, ez * (3 + np.log(V + 1)), "logp grad")
    return lp, lse, ent, out


def check_distill(a, W, ids, scores, weight, temperature):
    r, w = f64(a), f64(W)
    ez = logit_error(r, w, temperature)
    args = (a.to(DEV), W.to(DEV), ids.to(DEV), scores.to(DEV))
    cw = None if weight is None else weight.to(DEV)
    loss, grad = LL.ll_distill(*args, temperature=temperature, weight=cw)
    alone, none = LL.ll_distill(*args, temperature=temperature, weight=cw, grad=False)
    rl, dz, size = O.distill(r, w, ids.numpy(), f64(scores), temperature, f64(weight))
    bound = temperature ** 2 * 2 * ez + 1e-6 * np.abs(rl)
    assert none is None
    assert np.all(np.abs(f64(loss) - rl) <= bound) and np.all(np.abs(f64(alone) - rl) <= bound), float(np.max(np.abs(f64(loss) - rl) / bound))
    grad_close(grad, dz, size, w, ez, "distill grad")
    return loss, grad


@pytest.mark.parametrize("N,d,V,k", SIZES)
@pytest.mark.parametrize("temperature", [1.0, 0.7])
def test_logp_against_the_oracle(N, d, V, k, temperature):
    say(f"logp N={N} d={d} V={V} k={k} T={temperature}")
    a, W, ids, g = inputs(N, d, V, k)
    check_logp(a, W, ids, g, temperature, entropy=temperature != 1.0 or k % 2 == 0)


@pytest.mark.parametrize("N,d,V,k", SIZES)
@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_distill_against_the_oracle(N, d, V, k, temperature):
    say(f"distill N={N} d={d} V={V} k={k} T={temperature}")
    a, W, ids, g = inputs(N, d, V, k)
    scores = 3 * torch.randn((N, k), generator=g)
    weight = torch.rand((N,), generator=g) if temperature != 1.0 else None
    if N > 2:
        ids[N // 2] = -1                                        # a row without a teacher
        scores[1] = -float("inf")                               # another
        if weight is not None:
            weight[0] = 0.0
    loss, grad = check_distill(a, W, ids, scores, weight, temperature)
    if N > 2:
        dead = [1, N // 2] + ([0] if weight is not None else [])
        assert not grad[dead].any() and not loss[[1, N // 2]].any()


@pytest.mark.parametrize("spread,temperature", [(300.0, 1.0), (2000.0, 0.25), (300.0, 50.0)])
def test_logits_far_apart(spread, temperature):
    """Nearly all of the probability on a token or two, logits of hundreds; and flattened by the temperature."""
    say(f"logits far apart, {spread} T={temperature}")
    N, d, V, k = 70, 512, 1300, 6
    a, W, ids, g = inputs(N, d, V, k)
    a = (a.float() * (1 + spread * torch.rand((N, 1), generator=g) / 20)).to(torch.bfloat16)
    check_logp(a, W, ids, g, temperature)
    check_distill(a, W, ids, 5 * torch.randn((N, k), generator=g), None, temperature)


@pytest.mark.parametrize("N,d,V", [(1, 256, 3000), (4, 1024, 2000), (3, 5120, 700), (70, 512, 3000), (300, 264, 2000)])
@pytest.mark.parametrize("gap", [20.0, 300.0])
def test_lists_far_below_the_most_likely_token(N, d, V, gap):
    """Every second row has its probability on a token that its list does not name, up to hundreds of nats above those that it does: the
    exponents' reference, which starts from the list, has to move, in the middle of the vocabulary."""
    say(f"lists far below N={N} d={d} V={V} gap={gap}")
    a, W, ids, g = inputs(N, d, V, 5, spread=1.0)
    top = V // 2 + 7
    ids = torch.where((ids == top) | (ids < 0) | (ids >= V), (ids.abs() + 1) % (V // 4), ids).to(torch.int32)
    W[top] = (0.02 * torch.sign(W[top].float())).to(torch.bfloat16)       # of length 0.02 sqrt(d)
    a = a.float()
    a[::2] += gap / (0.0004 * d) * W[top].float()                          # its logit: gap and some
    a = a.to(torch.bfloat16)
    check_distill(a, W, ids, torch.randn((N, 5), generator=g), torch.rand((N,), generator=g) + 0.1, 1.0)
    check_logp(a, W, ids, g, 1.0)


@pytest.mark.parametrize("N,d,V,k", [(1, 256, 300, 2), (4, 1024, 777, 3), (3, 5120, 130, 2), (40, 136, 900, 5), (300, 264, 1001, 3)])
@pytest.mark.parametrize("power", [-60, 40, 100])
def test_gradients_of_any_size(N, d, V, k, power):
    """The gradient is linear in what it starts from, and a power of two changes no rounding: the same bits, but for the exponent.  (The
    columns past the vocabulary meet it too.)"""
    say(f"gradients times 2^{power} N={N} d={d} V={V}")
    a, W, ids, g = inputs(N, d, V, k)
    ca, cW, cids = a.to(DEV), W.to(DEV), ids.to(DEV)
    _, lse, ent = LL.ll_logp(ca, cW, cids)
    g_logp, g_ent = torch.randn((N, k), generator=g).to(DEV), torch.randn((N,), generator=g).to(DEV)
    plain = LL.ll_logp_grad(ca, cW, cids, lse, ent, g_logp, g_ent)
    scaled = LL.ll_logp_grad(ca, cW, cids, lse, ent, g_logp * 2.0 ** power, g_ent * 2.0 ** power)
    assert torch.isfinite(plain).all()
    # (what underflows on its way has no influence on a value of this size)
    torch.testing.assert_close(scaled.double(), plain.double() * 2.0 ** power, rtol=0, atol=2.0 ** power * 1e-12)


def test_nothing_of_a_masked_row_matters():
    say("masked rows of NaN and infinities")
    N, d, V, k = 40, 136, 900, 5
    a, W, ids, g = inputs(N, d, V, k)
    scores, weight = torch.randn((N, k), generator=g), torch.rand((N,), generator=g)
    ids[7], weight[9] = -1, 0.0
    loss, grad = check_distill(a, W, ids, scores, weight, 1.0)
    g_logp, lse = torch.randn((N, k), generator=g), None
    g_logp[7], g_logp[9] = 0.0, 0.0
    _, lse, ent = LL.ll_logp(a.to(DEV), W.to(DEV), ids.to(DEV))
    out = LL.ll_logp_grad(a.to(DEV), W.to(DEV), ids.to(DEV), lse, ent, g_logp.to(DEV))
    bad = a.clone()
    bad[7, 3], bad[9], scores[7] = float("nan"), float("inf"), float("nan")
    loss2, grad2 = LL.ll_distill(bad.to(DEV), W.to(DEV), ids.to(DEV), scores.to(DEV), weight=weight.to(DEV))
    assert torch.equal(grad2, grad) and not grad[7].any() and not grad[9].any() and loss2[7] == 0 and torch.isnan(loss2[9])
    keep = [r for r in range(N) if r != 9]
    assert torch.equal(loss2[keep], loss[keep])
    lse2 = lse.clone()
    lse2[7] = lse2[9] = float("nan")
    out2 = LL.ll_logp_grad(bad.to(DEV), W.to(DEV), ids.to(DEV), lse2, ent, g_logp.to(DEV))
    assert torch.equal(out, out2) and not out[7].any() and not out[9].any()


def test_a_row_that_is_no_number_stays_by_itself():
    say("a row of NaN among others")
    N, d, V, k = 300, 192, 1000, 3
    a, W, ids, g = inputs(N, d, V, k)
    scores = torch.randn((N, k), generator=g)
    lp, lse, ent, out = check_logp(a, W, ids, torch.Generator().manual_seed(5), 1.0)
    loss, grad = check_distill(a, W, ids, scores, None, 1.0)
    a[100, 7], a[101, 0] = float("nan"), float("inf")
    ca, cW, cids = a.to(DEV), W.to(DEV), ids.to(DEV)
    got = LL.ll_logp(ca, cW, cids)
    g_logp = torch.randn((N, k), generator=torch.Generator().manual_seed(5))
    g = torch.Generator().manual_seed(5)
    torch.randn((N, k), generator=g)
    got += (LL.ll_logp_grad(ca, cW, cids, got[1], got[2], g_logp.to(DEV), torch.randn((N,), generator=g).to(DEV)),)
    got += LL.ll_distill(ca, cW, cids, scores.to(DEV))
    others = [r for r in range(N) if r not in (100, 101)]
    for x, y in zip(got, (lp, lse, ent, out, loss, grad)):
        assert torch.equal(x[others].nan_to_num(7.0), y[others].nan_to_num(7.0))
        assert torch.isnan(x[[100, 101]].float()).all()


@pytest.mark.parametrize("N,d,V,k", [(5, 72, 700, 3), (600, 256, 3000, 8)])
def test_the_same_bits_twice_and_from_any_workspace(N, d, V, k):
    say(f"again, other workspaces N={N} d={d} V={V}")
    a, W, ids, g = inputs(N, d, V, k)
    ca, cW, cids, scores = a.to(DEV), W.to(DEV), ids.to(DEV), torch.randn((N, k), generator=g).to(DEV)
    g_logp, g_ent = torch.randn((N, k), generator=g).to(DEV), torch.randn((N,), generator=g).to(DEV)
    runs = []
    for fill in (0, 255, 127):
        ws = [torch.full((size(N, d, V, k),), fill, dtype=torch.uint8, device=DEV)
              for size in (LL.ll_logp_workspace_bytes, LL.ll_logp_grad_workspace_bytes, LL.ll_distill_workspace_bytes)]
        lp = LL.ll_logp(ca, cW, cids, workspace=ws[0])
        runs.append([*lp, LL.ll_logp_grad(ca, cW, cids, lp[1], lp[2], g_logp, g_ent, workspace=ws[1]),
                     *LL.ll_distill(ca, cW, cids, scores, workspace=ws[2])])
    for other in runs[1:]:
        for x, y in zip(runs[0], other):
            assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))


def test_the_last_rows_of_a_pass_of_long_rows():
    """P of a pass is more than 2^31 bytes apart at its ends: the last rows' gradients are those of a call of them alone, but for the order of
    the slices' sums."""
    say("rows far apart in the workspace")
    N, d, V, k = 1800, 64, 700001, 2
    g = torch.Generator(device=DEV).manual_seed(2)
    W = (0.1 * torch.randn((V, d), generator=g, device=DEV)).to(torch.bfloat16)
    a = torch.randn((N, d), generator=g, device=DEV).to(torch.bfloat16)
    ids = torch.randint(0, V, (N, k), generator=g, device=DEV, dtype=torch.int32)
    ids[:, 0] = V - 1
    scores = torch.randn((N, k), generator=g, device=DEV)
    loss, grad = LL.ll_distill(a, W, ids, scores)
    few, rest = LL.ll_distill(a[-20:].contiguous(), W, ids[-20:].contiguous(), scores[-20:].contiguous())
    torch.testing.assert_close(loss[-20:], few, rtol=1e-5, atol=1e-5)
    torch.testing.assert_close(grad[-20:].float(), rest.float(), rtol=2 ** -7, atol=2 ** -7 * float(rest.float().abs().mean()))


def test_no_rows():
    say("no rows")
    e, W = torch.empty((0, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((10, 64), dtype=torch.bfloat16, device=DEV)
    ids, f = torch.empty((0, 3), dtype=torch.int32, device=DEV), torch.empty((0, 3), device=DEV)
    lp, lse, ent = LL.ll_logp(e, W, ids)
    assert lp.shape == (0, 3) and lse.shape == ent.shape == (0,)
    assert LL.ll_logp_grad(e, W, ids, lse, ent, f).shape == (0, 64)
    loss, grad = LL.ll_distill(e, W, ids, f)
    assert loss.shape == (0,) and grad.shape == (0, 64)


def test_on_another_stream_and_in_a_graph():
    say("on a stream of its own, and captured")
    N, d, V, k = 200, 192, 3000, 4
    a, W, ids, g = inputs(N, d, V, k)
    ca, cW, cids, scores = a.to(DEV), W.to(DEV), ids.to(DEV), torch.randn((N, k), generator=g).to(DEV)
    g_logp, g_ent = torch.randn((N, k), generator=g).to(DEV), torch.randn((N,), generator=g).to(DEV)

    def everything(stream=None):
        lp = LL.ll_logp(ca, cW, cids, stream=stream)
        return [*lp, LL.ll_logp_grad(ca, cW, cids, lp[1], lp[2], g_logp, g_ent, stream=stream), *LL.ll_distill(ca, cW, cids, scores, stream=stream)]

    eager = everything()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = everything(side)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(eager, there):
        assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = everything()
    for turn in range(3):
        ca.copy_(ca.flip(0))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(captured, everything()):
            assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0)), turn


def test_gradients_are_the_slope_of_the_calls_themselves():
    """A step along a direction changes the returned loss as the returned gradient says: the loss is fp32, so the step is made large and
    central, of rows whose bf16 values the step keeps exact."""
    say("slopes")
    N, d, V, k = 64, 256, 900, 4
    a, W, ids, g = inputs(N, d, V, k)
    a = (torch.round(a.float() * 32) / 32).to(torch.bfloat16)           # multiples of 1/32 below 8: a step of 1/32 up or down is exact
    step = (torch.randint(0, 2, (N, d), generator=g).float() * 2 - 1) / 32
    a = a.float().clamp(-3, 3)
    scores, ids = torch.randn((N, k), generator=g), ids.abs() % V
    up, down = ((a + s * step).to(torch.bfloat16).to(DEV) for s in (1, -1))
    mid, cW, cids = a.to(torch.bfloat16).to(DEV), W.to(DEV), ids.to(torch.int32).to(DEV)
    cs = scores.to(DEV)
    slope = (f64(LL.ll_distill(up, cW, cids, cs, grad=False)[0]) - f64(LL.ll_distill(down, cW, cids, cs, grad=False)[0])) / 2
    grad = f64(LL.ll_distill(mid, cW, cids, cs)[1])
    # along the step: bf16 rounding of 256 terms (random), and the third derivative of a log-sum-exp, at most |s|^3 / 6 with
    # |s| the spread of the logits' change, sqrt(256) / 32 * 0.02 * 4 < 0.05
    bound = 8 * 2.0 ** -9 * np.sqrt(np.sum((grad / 32) ** 2, axis=1)) + 0.05 ** 3 + 1e-5
    assert np.all(np.abs(np.sum(grad * f64(step), axis=1) - slope) <= bound)
    lp, lse, ent = LL.ll_logp(mid, cW, cids)
    g_logp = torch.randn((N, k), generator=g)
    grad = f64(LL.ll_logp_grad(mid, cW, cids, lse, ent, g_logp.to(DEV)))
    value = lambda x: np.sum(f64(LL.ll_logp(x, cW, cids)[0]) * f64(g_logp), axis=1)
    bound = 8 * 2.0 ** -9 * np.sqrt(np.sum((grad / 32) ** 2, axis=1)) + (0.05 ** 3 + 1e-5) * np.sum(np.abs(f64(g_logp)), axis=1)
    assert np.all(np.abs(np.sum(grad * f64(step), axis=1) - (value(up) - value(down)) / 2) <= bound)
