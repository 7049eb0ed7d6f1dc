"""Learning from answers under autograd, the optimiser, and all of it together as a training step."""
import numpy as np
import pytest
import torch

from paper_2604_06483_amd import binding as LL
from paper_2604_06483_amd import tune
from tests.conftest import say
from tests.test_gpu_learn import f64, inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def answers(N, d, V, seed=0):
    a, W, ids, g = inputs(N, d, V, 1, seed=seed)
    return a.to(DEV), W.to(DEV), ids[:, 0].contiguous().clamp(0, V - 1).to(DEV), g


def test_autograd_passes_on_what_the_calls_return():
    say("autograd of answers")
    N, d, V, P = 40, 128, 900, 4
    rows, W, ids, g = answers(N, d, V)
    A, old, weight = (torch.randn((N,), generator=g).to(DEV) for _ in range(3))
    old = LL.ll_policy(rows, W, ids, A, grad=False)[1] + 0.1 * old
    weight = weight.abs()
    leaf = rows.clone().requires_grad_()
    loss, logp = tune.policy(leaf, W, ids, A, old, ref_logp=old, weight=weight, kl=0.1, temperature=0.5)
    loss.sum().backward()
    want = LL.ll_policy(rows, W, ids, A, old, ref_logp=old, weight=weight, kl=0.1, temperature=0.5)
    assert torch.equal(loss, weight * want[0]) and torch.equal(logp, want[1]) and torch.equal(leaf.grad, want[2])
    offsets = torch.tensor([0, 5, 9, 9, 20, 22, 30, 31, 38], dtype=torch.int32, device=DEV)
    factor = torch.tensor([1.0, 2.0, 0.5, 4.0], device=DEV)        # (powers of two round nothing again)
    leaf = rows.clone().requires_grad_()
    loss, score, logp = tune.preference(leaf, W, ids, offsets, ref_logp=old, weight=weight[:P])
    (factor * loss).sum().backward()
    want = LL.ll_preference(rows, W, ids, offsets, ref_logp=old, weight=weight[:P].contiguous())
    assert torch.equal(loss, weight[:P] * want[0]) and torch.equal(score, want[1]) and torch.equal(logp, want[2])
    by = torch.zeros((N,), device=DEV)
    for j in range(P):
        by[int(offsets[2 * j]):int(offsets[2 * j + 2])] = factor[j]
    assert torch.equal(leaf.grad, (by[:, None] * want[3]).to(torch.bfloat16)) and not leaf.grad[38:].any()


def test_gradients_are_the_slope_of_the_calls_themselves():
    """A step along a direction, of rows whose bf16 values it keeps exact, changes the returned loss as the returned gradient says."""
    say("slopes of answers")
    N, d, V = 64, 256, 900
    a, W, ids, g = inputs(N, d, V, 1)
    ids = ids[:, 0].contiguous().clamp(0, V - 1)
    a = (torch.round(a.float() * 32) / 32).clamp(-3, 3)
    step = (torch.randint(0, 2, (N, d), generator=g).float() * 2 - 1) / 32
    up, down, mid = ((a + s * step).to(torch.bfloat16).to(DEV) for s in (1, -1, 0))
    W, ids, A = W.to(DEV), ids.to(DEV), torch.randn((N,), generator=g).to(DEV)
    _, at, _ = LL.ll_policy(mid, W, ids, A, grad=False)
    ref = at + 0.3 * torch.randn((N,), generator=g).to(DEV)
    # no bound, so that the loss is smooth along the step; the ratio and e^q are near 1
    call = lambda x, grad: LL.ll_policy(x, W, ids, A, at, ref_logp=ref, clip=(1.0, float("inf")), kl=0.5, grad=grad)  # noqa: E731
    slope = (f64(call(up, False)[0]) - f64(call(down, False)[0])) / 2
    grad = f64(call(mid, True)[2])
    # along the step: bf16 rounding of 256 terms (random), and third differences: the logits' change has a spread below 0.05 (see the learning
    # calls' test), l's is D of at most its six standard deviations 0.1, and the third derivative of e^l is 1, times |A| + kl e^q
    bound = 8 * 2.0 ** -9 * np.sqrt(np.sum((grad / 32) ** 2, axis=1)) + (np.abs(f64(A)) + 0.5 * np.exp(np.abs(f64(ref - at)))) * (0.1 ** 3 + 1e-5)
    assert np.all(np.abs(np.sum(grad * f64(step), axis=1) - slope) <= bound)
    offsets = torch.arange(0, N + 1, 8, dtype=torch.int32, device=DEV)
    call = lambda x, grad: LL.ll_preference(x, W, ids, offsets, beta=0.5, grad=grad)  # noqa: E731
    slope = (f64(call(up, False)[0]) - f64(call(down, False)[0])) / 2
    grad = f64(call(mid, True)[3])
    got = np.sum((grad * f64(step)).reshape(4, -1), axis=1)
    # h changes by at most beta times 16 rows' 0.1, in root: 0.2; the third derivative of log sigmoid is below 0.1
    bound = 8 * 2.0 ** -9 * np.sqrt(np.sum((grad / 32).reshape(4, -1) ** 2, axis=1)) + 0.1 * 0.2 ** 3 + 0.5 * 16 * (0.05 ** 3 + 1e-5)
    assert np.all(np.abs(got - slope) <= bound), (got, slope, bound)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_optimiser_is_the_call(bits, dtype):
    """Groups, clipping and saved states: the bits of ll_grad_norm and ll_adamw called by hand."""
    say(f"optimiser, {bits} bits, {dtype}")
    g = torch.Generator(device=DEV).manual_seed(5)
    sizes = [(300, 7), (5,), (1000,)]
    start = [torch.randn(s, generator=g, device=DEV).to(dtype) for s in sizes]
    grads = [[torch.randn(s, generator=g, device=DEV).to(dtype) for s in sizes] for _ in range(4)]
    params = [torch.nn.Parameter(x.clone()) for x in start]
    copy = {params[0]: torch.empty(sizes[0], dtype=torch.bfloat16, device=DEV)} if dtype == torch.float32 else None

    def make(ps, copies=None):
        return tune.AdamW([{"params": ps[:2]}, {"params": ps[2:], "lr": 0.5, "weight_decay": 0.0}], lr=1e-2, bits=bits, max_norm=1.5, seed=3, copies=copies)

    opt = make(params, copy)

    def zeros(size):
        if bits == 32:
            return [torch.zeros(size, device=DEV), torch.zeros(size, device=DEV), None, None]
        codes = [torch.zeros(size, dtype=torch.uint8, device=DEV).view(t) for t in (torch.float8_e4m3fn, torch.float8_e5m2)]
        return codes + [torch.zeros((-(-int(np.prod(size)) // 256),), device=DEV) for _ in range(2)]

    hand = [x.clone() for x in start]
    state = [zeros(s) for s in sizes]
    for t in range(4):
        if t == 2:                                        # saved and loaded by another
            other = [torch.nn.Parameter(p.detach().clone()) for p in params]
            saved, params, opt = opt.state_dict(), other, make(other)
            opt.load_state_dict(saved)
        for p, x in zip(params, grads[t]):
            p.grad = x.clone()
        opt.step()
        norm = LL.ll_grad_norm(grads[t])
        assert torch.equal(opt.norm, norm)
        for at, (i, j) in enumerate(((0, 2), (2, 3))):
            many = LL.TensorList(grads[t][i:j], hand[i:j], *[[s[k] for s in state[i:j]] for k in range(4)])
            LL.ll_adamw(many, t + 1, rate=(1e-2, 0.5)[at], decay=(0.01, 0.0)[at], norm=norm, max_norm=1.5, seed=3 + at)
        for p, x in zip(params, hand):
            assert torch.equal(p.detach(), x), t
        if copy is not None and t < 2:
            assert torch.equal(copy[params[0]], params[0].to(torch.bfloat16))


def test_the_optimiser_says_that_it_is_not_captured():
    say("optimiser under capture")
    p = torch.nn.Parameter(torch.ones((8,), device=DEV))
    p.grad = torch.ones_like(p)
    opt = tune.AdamW([p])
    opt.step()
    before = p.detach().clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="clock"):
            opt.step()
        scratch = before + 1                              # (a graph of something)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(p.detach(), before) and torch.equal(scratch, before + 1)


@pytest.mark.parametrize("bits", [32, 8])
def test_answers_train_a_translator(bits):
    """The whole step, rows to parameters, from pairs and from sampled tokens: it runs, everything stays finite, every parameter moves, and
    the reference's own scores are 0 before the first."""
    say(f"answers train a translator, {bits} bits")
    inner, last, gamma, W = tune.synthetic_layers(96, 128, 700, DEV)
    ids = LL.ll_project(last, gamma, W, 1e-5, 1)[0].reshape(-1)
    ids[90:] = -1
    offsets = torch.arange(0, 97, 12, dtype=torch.int32, device=DEV)
    t = tune.Translator(128, gamma, 1e-5)
    start = [p.detach().clone() for p in t.parameters()]
    got = tune.fit_preference(t, inner, W, ids, offsets, steps=4, mean=True, bits=bits)
    assert len(got.losses) == 4 and np.allclose(got.losses[0], np.log(2), rtol=1e-5) and bool(torch.isfinite(got.scores).all()) and got.scores.shape == (4, 2)
    assert all(torch.isfinite(p).all() and not torch.equal(p, q) for p, q in zip(t.parameters(), start))
    t = tune.Translator(128, gamma, 1e-5)
    losses = tune.fit_policy(t, inner, W, ids, torch.randn((96,), device=DEV), updates=3, kl=0.1, bits=bits)
    assert len(losses) == 3 and np.all(np.isfinite(losses))
    assert all(torch.isfinite(p).all() and not torch.equal(p, q) for p, q in zip(t.parameters(), start))


def test_fit_takes_another_optimiser():
    say("fit with the library's step")
    inner, last, gamma, W = tune.synthetic_layers(64, 128, 500, DEV)
    result = tune.fit(tune.Translator(128, gamma, 1e-5), inner, last, W, k=4, steps=3, optimiser=lambda ps: tune.AdamW(ps, lr=1e-3, bits=8, max_norm=1.0))
    assert len(result.losses) == 3 and np.all(np.isfinite(result.losses))


def test_a_second_derivative_is_refused():
    say("autograd of answers, twice")
    rows, W, ids, g = answers(12, 64, 200)
    rows.requires_grad_()
    offsets = torch.tensor([0, 4, 12], dtype=torch.int32, device=DEV)
    factor = torch.ones((), device=DEV, requires_grad=True)
    for value in (tune.policy(rows, W, ids, torch.ones((12,), device=DEV))[0].sum(), tune.preference(rows, W, ids, offsets)[0].sum()):
        (grad,) = torch.autograd.grad(factor * value, rows, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            grad.float().sum().backward()


def test_gradients_in_a_graph():
    """Losses and gradients of both captured once, on inputs that are replaced between the replays: the eager ones each time."""
    say("autograd of answers in a graph")
    rows, W, ids, g = answers(60, 128, 700, seed=2)
    A, factor = torch.randn((60,), generator=g).to(DEV), torch.tensor([1.0, 2.0], device=DEV)
    offsets = torch.tensor([0, 20, 31, 31, 50], dtype=torch.int32, device=DEV)
    held = rows.clone().requires_grad_()

    def both(x):
        a = torch.autograd.grad(tune.policy(x, W, ids, A)[0].sum(), x)[0]
        b = torch.autograd.grad((factor * tune.preference(x, W, ids, offsets)[0]).sum(), x)[0]
        return a, b

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both(held)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = both(held)
    for turn in range(3):
        with torch.no_grad():
            held.copy_(torch.roll(rows, turn, 0))
            factor.mul_(2.0)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(out, both(held.detach().clone().requires_grad_())):
            assert torch.equal(x, y), turn


def test_a_step_on_another_stream():
    say("optimiser on another stream")
    a, b = (torch.nn.Parameter(torch.ones((1000,), device=DEV)) for _ in range(2))
    one, two = tune.AdamW([a], lr=0.1, max_norm=1.0), tune.AdamW([b], lr=0.1, max_norm=1.0)
    s = torch.cuda.Stream()
    for t in range(3):
        a.grad = torch.full((1000,), 0.5 + t, device=DEV)
        b.grad = a.grad.clone()
        one.step()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            two.step()
        torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a.detach(), b.detach())
