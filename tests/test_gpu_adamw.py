"""ll_grad_norm and ll_adamw against the fp64 oracle, and the 8-bit states bit for bit against their definition."""
import numpy as np
import pytest
import torch

import oracle.step_oracle as O
from paper_2604_06483_amd import binding as LL
from tests.conftest import say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, E4M3, E5M2 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.float8_e5m2
EPS24 = 2.0 ** -24
# one element, around four, around a block, around a workgroup's four blocks, more
SIZES = [(1,), (3,), (4,), (5,), (255,), (256,), (257,), (1023,), (1024,), (1025,), (37, 41), (3, 1000, 7), (0,), (5000,)]


class Problem:
    """Tensors on the CPU and on the GPU, and their list."""

    def __init__(self, sizes, param=F32, grad=F32, eight=False, copy=False, seed=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        normal = lambda size: torch.randn(size, generator=g) * torch.exp(spread * torch.randn(size, generator=g))  # noqa: E731
        self.eight = eight
        self.p = [(0.1 * normal(s)).to(param) for s in sizes]
        self.g = [(1e-2 * normal(s)).to(grad) for s in sizes]
        self.m, self.v = [1e-3 * normal(s) for s in sizes], [1e-4 * normal(s).square() for s in sizes]
        self.ms = self.vs = None
        if eight:
            self.m8, self.v8, self.ms, self.vs = [], [], [], []
            for i, s in enumerate(sizes):
                w = O.words(np.arange(self.p[i].numel()), 7, 1, i)
                a, b, sm, sv = O.states8(self.m[i].reshape(-1).numpy(), self.v[i].reshape(-1).numpy(), w) if self.p[i].numel() else ([], [], [], [])
                bytes_ = lambda x: torch.tensor(np.asarray(x, dtype=np.uint8))  # noqa: E731
                self.m8.append(bytes_(a).view(E4M3).reshape(s))
                self.v8.append(bytes_(b).view(E5M2).reshape(s))
                self.ms.append(torch.tensor(np.asarray(sm), dtype=F32))
                self.vs.append(torch.tensor(np.asarray(sv), dtype=F32))
                by = lambda sc, n: sc.repeat_interleave(256)[:n]  # noqa: E731
                self.m[i] = (self.m8[i].float().reshape(-1) * by(self.ms[i], self.p[i].numel())).reshape(s)
                self.v[i] = (self.v8[i].float().reshape(-1) * by(self.vs[i], self.p[i].numel())).reshape(s)
        to = lambda of: None if of is None else [x.to(DEV) for x in of]  # noqa: E731
        self.dp, self.dg = to(self.p), to(self.g)
        self.dm, self.dv = (to(self.m8), to(self.v8)) if eight else (to(self.m), to(self.v))
        self.dms, self.dvs = to(self.ms), to(self.vs)
        self.copies = [torch.empty(s, dtype=BF16, device=DEV) for s in sizes] if copy else None
        self.list = LL.TensorList(self.dg, self.dp, self.dm, self.dv, self.dms, self.dvs, self.copies)


def f64(x):
    return x.double().cpu().numpy().reshape(-1)


def check_step(q, step=3, rate=1e-2, betas=(0.9, 0.999), eps=1e-8, decay=0.1, norm=None, max_norm=float("inf"), seed=11, ran=None):
    """Runs the step and checks every tensor."""
    dn = None if norm is None else torch.tensor([norm], dtype=F32, device=DEV)
    if ran is None:
        LL.ll_adamw(q.list, step, rate=rate, betas=betas, eps=eps, decay=decay, norm=dn, max_norm=max_norm, seed=seed)
    torch.cuda.synchronize()
    clip = 1.0 if norm is None or norm <= max_norm else float(np.float32(max_norm) / np.float32(norm))
    for i in range(len(q.p)):
        n = q.p[i].numel()
        if n == 0:
            continue
        p, g, m, v = f64(q.p[i]), f64(q.g[i]), f64(q.m[i]), f64(q.v[i])
        rp, rm, rv = O.adamw(p, g, m, v, step, rate, betas, eps, decay, norm, max_norm)
        g = g * clip
        # m' is two products and a sum of fp32, v' a square more, with the betas and the clipping rounded to fp32 too
        size_m, size_v = betas[0] * np.abs(m) + (1 - betas[0]) * np.abs(g), betas[1] * v + (1 - betas[1]) * g * g
        off_m, off_v = 6 * EPS24 * size_m + 1e-44, 8 * EPS24 * size_v + 1e-44
        # the quotient: its divisor to some last bits (a root, two products' roundings, a reciprocal), m' as above, rounded into p
        by = rate / (1 - betas[0] ** step) / (np.sqrt(rv / (1 - betas[1] ** step)) + eps)
        off_p = 4 * EPS24 * np.abs(p) + by * (off_m + 16 * EPS24 * size_m) + 2 * EPS24 * np.abs(rp)
        got = f64(q.dp[i])
        if q.p[i].dtype == BF16:                              # rounded to one of its two neighbours
            off_p = off_p + 2.0 ** -7 * np.abs(rp) + 1e-40
        assert np.all(np.abs(got - rp) <= off_p), (i, n, float(np.max(np.abs(got - rp) / off_p)))
        if q.copies is not None:
            assert torch.equal(q.copies[i], q.dp[i].to(BF16))
        if not q.eight:
            assert np.all(np.abs(f64(q.dm[i]) - rm) <= off_m) and np.all(np.abs(f64(q.dv[i]) - rv) <= off_v), (i, n)
            continue
        m32, v32 = O.moments32(q.g[i].float().numpy().reshape(-1), q.m[i].numpy().reshape(-1), q.v[i].numpy().reshape(-1), betas, clip)
        assert np.all(np.abs(m32 - rm) <= off_m) and np.all(np.abs(v32 - rv) <= off_v)
        a, b, sm, sv = O.states8(m32, v32, O.words(np.arange(n), seed, step, i))
        assert np.array_equal(f64(q.dms[i]), sm) and np.array_equal(f64(q.dvs[i]), sv), (i, n)
        got_a, got_b = (x.view(torch.uint8).cpu().numpy().reshape(-1) for x in (q.dm[i], q.dv[i]))
        assert np.array_equal(got_a, a), (i, n, int((got_a != a).sum()))
        assert np.array_equal(got_b, b), (i, n, int((got_b != b).sum()))


@pytest.mark.parametrize("param", [F32, BF16])
@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("eight", [False, True])
def test_a_step_of_every_kind(param, grad, eight):
    say(f"adamw {param} {grad} eight={eight}")
    check_step(Problem(SIZES, param, grad, eight, copy=param == F32, seed=1), norm=5.0, max_norm=1.5)
    check_step(Problem(SIZES[::-1], param, grad, eight, seed=2), step=1, decay=0.0, norm=5.0, max_norm=float("inf"))
    check_step(Problem(SIZES, param, grad, eight, seed=3, spread=3.0), step=10 ** 6, betas=(0.0, 0.5), eps=1e-3)


def test_more_tensors_than_a_launch_takes():
    say("adamw, 130 tensors")
    sizes = [(1 + 37 * i % 700,) for i in range(130)]
    for eight in (False, True):
        check_step(Problem(sizes, eight=eight, seed=4))


def test_kinds_mixed_in_one_list():
    say("adamw, mixed kinds")
    parts = [Problem([(300,), (5, 70)], p, g, e, seed=20 + k) for k, (p, g, e) in enumerate((a, b, c) for a in (F32, BF16) for b in (F32, BF16) for c in (False, True))]
    order = [(k, i) for i in range(2) for k in range(8)]
    pick = lambda name: [getattr(parts[k], name)[i] if getattr(parts[k], name) is not None else None for k, i in order]  # noqa: E731
    whole = LL.TensorList(pick("dg"), pick("dp"), pick("dm"), pick("dv"), pick("dms"), pick("dvs"))
    LL.ll_adamw(whole, 3, rate=1e-2, decay=0.1, seed=11)
    for at, (k, i) in enumerate(order):                       # each as if alone, at its place in the list
        q = parts[k]
        n = q.p[i].numel()
        if q.eight:
            m32, v32 = O.moments32(q.g[i].float().numpy().reshape(-1), q.m[i].numpy().reshape(-1), q.v[i].numpy().reshape(-1), (0.9, 0.999))
            a, b, _, _ = O.states8(m32, v32, O.words(np.arange(n), 11, 3, at))
            assert np.array_equal(q.dm[i].view(torch.uint8).cpu().numpy().reshape(-1), a), at
            assert np.array_equal(q.dv[i].view(torch.uint8).cpu().numpy().reshape(-1), b), at
        else:
            check_step(Problem([(300,), (5, 70)], q.p[i].dtype, q.g[i].dtype, False, seed=20 + k))
            rp = O.adamw(f64(q.p[i]), f64(q.g[i]), f64(q.m[i]), f64(q.v[i]), 3, 1e-2, (0.9, 0.999), 1e-8, 0.1)[0]
            assert np.all(np.abs(f64(q.dp[i]) - rp) <= 1e-6 + 2.0 ** -7 * np.abs(rp) * (q.p[i].dtype == BF16) + 8 * EPS24 * np.abs(rp))


def test_bf16_parameters_are_rounded_without_bias():
    """A step of a 40th of a last bit, 4096 times: the mean of 4096 parameters moves as the steps say, where the nearest would stay."""
    say("adamw, bf16 parameters")
    n = 4096
    p, g = torch.ones((n,), dtype=BF16, device=DEV), torch.ones((n,), dtype=F32, device=DEV)
    m, v = torch.ones((n,), device=DEV), torch.ones((n,), device=DEV)
    steps, rate = 400, 2.0 ** -8 / 40                          # downwards from 1 a last bit is 2^-8
    many = LL.TensorList([g], [p], [m], [v])
    for t in range(steps):
        LL.ll_adamw(many, 10 ** 6 + t, rate=rate, betas=(0.5, 0.5), eps=1e-12, seed=5)
    # each element does `steps` roundings of variance at most 2^-16 / 40: the mean's standard deviation is 2^-8 sqrt(steps / 40 / n)
    moved, sigma = 1.0 - float(p.double().mean()), 2.0 ** -8 * (steps / 40 / n) ** 0.5
    assert abs(moved - steps * rate) <= 6 * sigma, (moved, steps * rate, sigma)


def test_8_bit_states_follow_their_averages():
    """Constant gradients: the mean over many elements of v is g^2 (1 - b2^t), of m g (1 - b1^t), though b2 moves v by less than a step of its code."""
    say("adamw, 8-bit averages")
    n, steps = 1 << 16, 300
    g = torch.full((n,), 0.3, device=DEV)
    zeros = lambda dtype: torch.zeros((n,), dtype=torch.uint8, device=DEV).view(dtype)  # noqa: E731
    m, v, ms, vs = zeros(E4M3), zeros(E5M2), torch.zeros((n // 256,), device=DEV), torch.zeros((n // 256,), device=DEV)
    many = LL.TensorList([g], [torch.zeros((n,), device=DEV)], [m], [v], [ms], [vs])
    for t in range(1, steps + 1):
        LL.ll_adamw(many, t, rate=1e-3, seed=6)
    got_m, got_v = ((x.double().reshape(-1, 256) * s.double()[:, None]).mean().item() for x, s in ((m, ms), (v, vs)))
    want_m, want_v = 0.3 * (1 - 0.9 ** steps), 0.09 * (1 - 0.999 ** steps)
    # a step adds a rounding's variance of at most (value / 4)^2 / 4 to v and a fourth of that to m, before what they average over forgets it:
    # at most 300 of them for v, 1 / (1 - 0.81) for m; the mean's is n times less
    off_v, off_m = 6 * 0.125 * want_v * (steps / n) ** 0.5, 6 * 0.0625 * want_m * (5.3 / n) ** 0.5
    assert abs(got_v - want_v) <= off_v and abs(got_m - want_m) <= off_m, (got_v, want_v, off_v, got_m, want_m, off_m)


@pytest.mark.parametrize("eight", [False, True])
def test_gradients_that_are_not_finite(eight):
    say("adamw, NaN and infinity")
    q = Problem([(1000,)], eight=eight, seed=8)
    clean = Problem([(1000,)], eight=eight, seed=8)
    at = [3, 300, 999]
    for i, bad in zip(at, (float("nan"), float("inf"), -float("inf"))):
        q.dg[0][i] = bad
    clean.dg[0][at] = 0.0
    clean_at = torch.ones((1000,), dtype=torch.bool)
    clean_at[at] = False
    # the norm says so, and then nothing happens
    norm = LL.ll_grad_norm(q.list)
    assert not torch.isfinite(norm).any()
    before = [x.clone().view(torch.uint8) for x in (q.dp[0], q.dm[0], q.dv[0])]
    LL.ll_adamw(q.list, 1, norm=norm, max_norm=1.0)
    assert all(torch.equal(x.view(torch.uint8), y) for x, y in zip((q.dp[0], q.dm[0], q.dv[0]), before))
    # without a norm, the element's own are lost
    LL.ll_adamw(q.list, 1)
    LL.ll_adamw(clean.list, 1)
    where = clean_at.to(DEV)
    assert torch.equal(q.dp[0][where], clean.dp[0][where]) and not torch.isfinite(q.dp[0][~where]).any()
    assert not torch.isfinite(q.dm[0].float()[~where]).any() and not torch.isfinite(q.dv[0].float()[~where]).any()
    assert torch.isfinite(q.dm[0].float()[where]).all() and torch.isfinite(q.dv[0].float()[where]).all()
    if eight:
        assert torch.isfinite(q.dms[0]).all() and torch.isfinite(q.dvs[0]).all()


def test_tiny_and_huge_values():
    """From where squares underflow to where they are near the largest number: nothing but what is NaN or infinite by the formula is."""
    say("adamw, tiny and huge")
    for size in (1e-30, 1e-20, 1e-10, 1e10, 1e18):
        for eight in (False, True):
            q = Problem([(512,)], eight=eight, seed=9)
            q.g = [size * torch.sign(x) * (1 + x.abs()) for x in q.g]
            q.m, q.v = [torch.zeros_like(x) for x in q.m], [torch.zeros_like(x) for x in q.v]
            for t in [q.dm[0], q.dv[0]] + ([q.dms[0], q.dvs[0]] if eight else []):
                t.view(torch.uint8).zero_()
            q.dg[0].copy_(q.g[0])
            check_step(q, step=1, eps=1e-8 if size > 1e-12 else 1e-15)


@pytest.mark.parametrize("eight", [False, True])
def test_captured_with_a_clock(eight):
    """A captured norm and step, replayed with other gradients and rates between: the eager steps' bits each time."""
    say(f"adamw in a graph eight={eight}")
    sizes = [(700,), (33, 31)]
    a, b = Problem(sizes, eight=eight, copy=True, seed=10), Problem(sizes, eight=eight, copy=True, seed=10)
    clock, rate = torch.zeros((4,), dtype=torch.int64, device=DEV), torch.full((1,), 1e-2, device=DEV)
    ws = torch.empty((LL.ll_grad_norm_workspace_bytes(a.list),), dtype=torch.uint8, device=DEV)
    norm = torch.empty((1,), device=DEV)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def body(stream=None):
        LL.ll_grad_norm(a.list, workspace=ws, stream=stream, out=norm)
        LL.ll_adamw(a.list, rate=99.0, decay=0.1, norm=norm, max_norm=0.5, seed=3, clock=clock, device_rate=rate, stream=stream)

    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        body(s)
    for t in range(1, 5):
        for i, g in enumerate(a.dg):
            g.mul_(0.7 + 0.2 * t)
            b.dg[i].copy_(g)
        rate.fill_(1e-2 / t)
        if t == 3:                                            # a step that is left out is not counted
            a.dg[0][5] = float("inf")
        graph.replay()
        torch.cuda.synchronize()
        if t == 3:
            a.dg[0][5] = b.dg[0][5]
            assert int(clock[0]) == 2
            graph.replay()
            torch.cuda.synchronize()
        want = LL.ll_grad_norm(b.list)
        LL.ll_adamw(b.list, t, rate=float(rate), decay=0.1, norm=want, max_norm=0.5, seed=3)
        torch.cuda.synchronize()
        assert int(clock[0]) == t and torch.equal(norm, want)
        for x, y in zip(a.dp + a.dm + a.dv + a.copies + (a.dms + a.dvs if eight else []), b.dp + b.dm + b.dv + b.copies + (b.dms + b.dvs if eight else [])):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), t


def test_other_gradients_and_another_stream():
    say("adamw, set_grads and a stream")
    q, r = Problem([(600,), (7, 9)], seed=12), Problem([(600,), (7, 9)], seed=12)
    other = [x.to(BF16) for x in q.dg]
    q.list.set_grads(other)
    q.g = [x.cpu() for x in other]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    LL.ll_adamw(q.list, 3, rate=1e-2, decay=0.1, seed=11, stream=s)
    s.synchronize()
    check_step(q, ran=True)
    with pytest.raises(ValueError):
        q.list.set_grads(other[:1])
    with pytest.raises(ValueError):
        q.list.set_grads([other[0], other[1].T.contiguous()])
    with pytest.raises(TypeError):
        q.list.set_grads([other[0], torch.zeros((9, 7), device=DEV).T])
    check_step(r)


def test_lists_that_are_refused():
    say("adamw, refusals")
    x, h = (lambda *s: torch.zeros(s, device=DEV)), torch.zeros((8,), dtype=BF16, device=DEV)
    m8, v8 = (torch.zeros((8,), dtype=torch.uint8, device=DEV).view(t) for t in (E4M3, E5M2))
    one = x(8)
    for error, args in ((ValueError, ([x(8)], [x(8)])), (ValueError, ([x(8)], [one], [x(8)], [one])), (ValueError, ([x(8), x(8)], [one, one], [x(8), x(8)], [x(8), x(8)])),
                        (ValueError, ([x(8)], [x(4)], [x(8)], [x(8)])), (TypeError, ([x(8)], [x(8)], [m8], [x(8)], [x(1)], [x(1)])),
                        (TypeError, ([x(8)], [x(8)], [m8], [v8])), (ValueError, ([x(8)], [x(8)], [m8], [v8], [x(2)], [x(1)])),
                        (ValueError, ([x(8)], [x(8)], [x(8)], [x(8)], [x(1)], None)), (ValueError, ([x(8)], [h], [x(8)], [x(8)], None, None, [h.clone()])),
                        (TypeError, ([x(8).double()],)), (TypeError, ([x(8, 8).T[:, :3]],))):
        with pytest.raises(error):
            LL.TensorList(*args)
    ok = LL.TensorList([x(8)], [x(8)], [x(8)], [x(8)])
    for kw in (dict(), dict(step=1, clock=torch.zeros((4,), dtype=torch.int64, device=DEV))):
        with pytest.raises(ValueError):
            LL.ll_adamw(ok, **kw)
    with pytest.raises(TypeError):
        LL.ll_adamw(LL.TensorList([x(8)]), 1)
    with pytest.raises(LL.LLError):
        LL.ll_adamw(ok, 0)
    with pytest.raises(LL.LLError):                            # a view that begins inside 16 bytes
        LL.ll_grad_norm([x(9)[1:]])


@pytest.mark.parametrize("sizes", [[(1,)], [(5,), (0,), (1000,)], [(100000,), (8191,), (8192,), (8193,)], [(3000000,)], [(50 + i,) for i in range(400)], [], [(0,)]])
def test_grad_norm(sizes):
    say(f"grad norm of {len(sizes)}")
    g = torch.Generator().manual_seed(len(sizes))
    grads = [(torch.randn(s, generator=g) * 10.0 ** (i % 9 - 4)).to(BF16 if i % 2 else F32).to(DEV) for i, s in enumerate(sizes)]
    got = LL.ll_grad_norm(grads)
    want = float(np.sqrt(sum(float(np.sum(f64(x) ** 2)) for x in grads)))
    # squares and sums in fp64, rounded once
    assert abs(float(got) - want) <= (2.0 ** -24 + 1e-12) * want
    assert torch.equal(got, LL.ll_grad_norm(grads))


def test_grad_norm_of_squares_that_fp32_does_not_hold():
    say("grad norm, 1e-30 and 1e30")
    for size in (1e-30, 1e30):
        x = torch.full((1000,), size, device=DEV)
        assert abs(float(LL.ll_grad_norm([x])) / (1000 ** 0.5 * float(x[0])) - 1) < 2.0 ** -23


def test_elements_past_32_bits():
    """One tensor of 2^32 + 1003 elements: its end is what the definition says of those elements."""
    n, k = 2 ** 32 + 1003, 1003 + 512
    say(f"adamw of {n} elements")
    zeros = lambda dtype: torch.zeros((n,), dtype=torch.uint8, device=DEV).view(dtype)  # noqa: E731
    p, g = torch.zeros((n,), dtype=BF16, device=DEV), torch.zeros((n,), dtype=BF16, device=DEV)
    m, v = zeros(E4M3), zeros(E5M2)
    blocks = (n + 255) // 256
    ms, vs = torch.zeros((blocks,), device=DEV), torch.zeros((blocks,), device=DEV)
    tail = (1e-2 * torch.randn((k,), generator=torch.Generator().manual_seed(1))).to(BF16)
    g[-k:] = tail.to(DEV)
    many = LL.TensorList([g], [p], [m], [v], [ms], [vs])
    want = float(np.sqrt(np.sum(f64(tail) ** 2)))
    assert abs(float(LL.ll_grad_norm(many)) - want) <= 2.0 ** -23 * want
    LL.ll_adamw(many, 1, rate=1e-2, seed=4)
    m32, v32 = O.moments32(tail.float().numpy(), np.zeros(k, dtype=np.float32), np.zeros(k, dtype=np.float32), (0.9, 0.999))
    a, b, sm, sv = O.states8(m32, v32, O.words(np.arange(n - k, n, dtype=np.uint64), 4, 1, 0))
    assert np.array_equal(m[-k:].view(torch.uint8).cpu().numpy(), a) and np.array_equal(v[-k:].view(torch.uint8).cpu().numpy(), b)
    assert np.array_equal(f64(ms[-6:]), sm) and np.array_equal(f64(vs[-6:]), sv)
    rp = O.adamw(np.zeros(k), f64(tail), np.zeros(k), np.zeros(k), 1, 1e-2, (0.9, 0.999), 1e-8, 0.0)[0]
    assert np.all(np.abs(f64(p[-k:]) - rp) <= (2.0 ** -7 + 2.0 ** -19) * np.abs(rp))
    assert not p[:-k].any() and not m[:-k].view(torch.uint8).any()
