"""Training through the lens: translators that bring an inner layer's states to what the last layer's lens reads out.

The raw logit lens (ll_project) applies the model's final norm and unembedding to states that were never meant for them.  A translator
per layer, x = h + scale gate (h A^T + b), learns what is missing from the model itself: its teacher is the last layer's own read-out,
the k most likely tokens that ll_project lists.  Nothing of the model changes.

`block_norm`, `token_logp`, `distill`, `policy` and `preference` are the library's calls with their gradients, for torch's autograd; `Translator` and
`fit` put them together:

    rows  -> product with A (torch) -> ll_block_norm -> ll_distill -> gradient of the normed rows -> ll_block_norm_grad -> A, b, gate

`fit_policy` and `fit_preference` train one on answers instead: sampled tokens with their advantages, or pairs of which one is preferred.  `AdamW` is
the library's step over all parameters at once, with states in 32 or in 8 bits.

    python -m paper_2604_06483_amd.tune            # a small synthetic model on the GPU
"""
from __future__ import annotations

from dataclasses import dataclass

import torch
from torch.autograd.function import once_differentiable

from . import binding as LL


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, y, gamma, gate, gamma_y, eps, scale):
        ctx.types = [None if p is None else p.dtype for p in (gamma, gate, gamma_y)]
        gamma, gate, gamma_y = (p.to(torch.bfloat16) if t == torch.float32 else p for p, t in zip((gamma, gate, gamma_y), ctx.types))
        ctx.save_for_backward(hidden, y, gamma, gate, gamma_y)
        ctx.eps, ctx.scale = eps, scale
        ctx.set_materialize_grads(False)
        return LL.ll_block_norm(hidden, y, gamma, eps, gate=gate, scale=scale, gamma_y=gamma_y)

    @staticmethod
    @once_differentiable
    def backward(ctx, g_hidden, g_normed):
        hidden, y, gamma, gate, gamma_y = ctx.saved_tensors
        g_hidden = None if g_hidden is None else g_hidden.contiguous()
        g_normed = torch.zeros_like(hidden) if g_normed is None else g_normed.contiguous()
        d_hidden, d_y, d_gate, d_gamma_y, d_gamma = LL.ll_block_norm_grad(hidden, y, gamma, ctx.eps, g_hidden, g_normed, gate=gate,
                                                                          scale=ctx.scale, gamma_y=gamma_y)
        d_gamma, d_gate, d_gamma_y = (None if t is None else g.to(t) for g, t in zip((d_gamma, d_gate, d_gamma_y), ctx.types))
        return d_hidden, d_y.reshape(y.shape), d_gamma, d_gate, d_gamma_y, None, None


class _TokenLogp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rows, W_U, ids, temperature):
        logp, lse, entropy = LL.ll_logp(rows, W_U, ids, temperature=temperature)
        ctx.save_for_backward(rows, W_U, ids, lse, entropy)
        ctx.temperature = temperature
        ctx.set_materialize_grads(False)
        return logp, entropy

    @staticmethod
    @once_differentiable
    def backward(ctx, g_logp, g_entropy):
        rows, W_U, ids, lse, entropy = ctx.saved_tensors
        g_logp = torch.zeros(ids.shape, dtype=torch.float32, device=rows.device) if g_logp is None else g_logp.contiguous()
        g_entropy = None if g_entropy is None else g_entropy.contiguous()
        grad = LL.ll_logp_grad(rows, W_U, ids, lse, entropy, g_logp, g_entropy, temperature=ctx.temperature)
        return grad, None, None, None


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rows, W_U, teacher_ids, teacher_scores, temperature, weight):
        loss, grad = LL.ll_distill(rows, W_U, teacher_ids, teacher_scores, temperature=temperature, weight=weight, grad=ctx.needs_input_grad[0])
        ctx.save_for_backward(grad, loss if ctx.needs_input_grad[5] else None)
        return loss if weight is None else (weight * loss).masked_fill(weight == 0, 0.0)   # (a row of weight 0 may hold anything)

    @staticmethod
    @once_differentiable
    def backward(ctx, g_loss):
        grad, loss = ctx.saved_tensors
        d_rows = None if grad is None else (g_loss.reshape(grad.shape[:-1] + (1,)) * grad).to(grad.dtype)
        return d_rows, None, None, None, None, None if loss is None else g_loss * loss


class _Policy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rows, W_U, ids, advantage, old_logp, weight, options):
        loss, logp, grad = LL.ll_policy(rows, W_U, ids, advantage, old_logp, weight=weight, grad=ctx.needs_input_grad[0], **options)
        ctx.save_for_backward(grad, loss.reshape(weight.shape) if ctx.needs_input_grad[5] else None)
        ctx.mark_non_differentiable(logp)
        ctx.set_materialize_grads(False)
        return loss if weight is None else (weight.reshape(-1) * loss).masked_fill(weight.reshape(-1) == 0, 0.0), logp

    @staticmethod
    @once_differentiable
    def backward(ctx, g_loss, _):
        grad, loss = ctx.saved_tensors
        if g_loss is None:
            return (None,) * 7
        d_rows = None if grad is None else (g_loss.reshape(grad.shape[:-1] + (1,)) * grad).to(grad.dtype)
        return d_rows, None, None, None, None, None if loss is None else g_loss.reshape(loss.shape) * loss, None


class _Preference(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rows, W_U, ids, offsets, weight, options):
        loss, score, logp, grad = LL.ll_preference(rows, W_U, ids, offsets, weight=weight, grad=ctx.needs_input_grad[0], **options)
        ctx.save_for_backward(grad, loss.reshape(weight.shape) if ctx.needs_input_grad[4] else None, offsets)
        ctx.mark_non_differentiable(score, logp)
        ctx.set_materialize_grads(False)
        return loss if weight is None else (weight.reshape(-1) * loss).masked_fill(weight.reshape(-1) == 0, 0.0), score, logp

    @staticmethod
    @once_differentiable
    def backward(ctx, g_loss, *_):
        grad, loss, offsets = ctx.saved_tensors
        if g_loss is None:
            return (None,) * 6
        d_rows = None
        if grad is not None:
            # the pair of every row: its sequence is the first that ends behind it; rows of none have no gradient
            flat = grad.reshape(-1, grad.shape[-1])
            at = torch.arange(flat.shape[0], dtype=torch.int32, device=grad.device)
            pair = torch.searchsorted(offsets[1:].contiguous(), at, right=True) // 2
            inside = pair < g_loss.shape[0]
            by = torch.where(inside, torch.cat([g_loss, g_loss.new_zeros((1,))])[pair], 0.0)
            d_rows = (by[:, None] * flat).to(grad.dtype).reshape(grad.shape)
        return d_rows, None, None, None, None if loss is None else g_loss.reshape(loss.shape) * loss, None


def _no_gradient(**tensors):
    """What the library has no gradient of is refused where autograd would be asked for one: without it a training step would miss a term."""
    if torch.is_grad_enabled():
        for name, t in tensors.items():
            if t is not None and t.requires_grad:
                raise ValueError(f"{name} gets no gradient: pass it detached")


def block_norm(hidden, y, gamma, eps, *, gate=None, scale=1.0, gamma_y=None):
    """ll_block_norm, differentiable in hidden, y, gamma, gate and gamma_y: (x, gamma x / rms(x)).

    gamma, gate and gamma_y may be fp32: they are rounded to bf16 for the call, and what all rows share gets the call's fp32 sums as they are.
    The gradient of a parameter in bf16 is rounded to it, as autograd's types demand."""
    return _BlockNorm.apply(hidden, y, gamma, gate, gamma_y, eps, scale)


def token_logp(rows, W_U, ids, *, temperature=1.0):
    """ll_logp, differentiable in the rows: (log-probabilities of the listed tokens, entropy).  W_U gets no gradient: detached, or an error."""
    _no_gradient(W_U=W_U)
    return _TokenLogp.apply(rows, W_U, ids, temperature)


def distill(rows, W_U, teacher_ids, teacher_scores, *, temperature=1.0, weight=None):
    """ll_distill, differentiable in the rows and the weight: weight times every row's loss.  The rows' gradient is formed with the loss, in one
    call, in bf16: give the weights here (1 / N for a mean), and sum (an incoming gradient other than a power of two rounds it again).  W_U and the
    teacher get no gradient: detached, or an error."""
    _no_gradient(W_U=W_U, teacher_scores=teacher_scores)
    return _Distill.apply(rows, W_U, teacher_ids, teacher_scores, temperature, weight)


def policy(rows, W_U, ids, advantage, old_logp=None, *, ref_logp=None, weight=None, clip=(0.2, 0.2), kl=0.0, temperature=1.0):
    """ll_policy, differentiable in the rows and the weight: (weight times every row's loss, the tokens' log-probabilities, which have no
    gradient here).  The rows' gradient is formed with the loss, as in `distill`: give the weights here, and sum.  W_U, the advantages and the
    other policies' log-probabilities get no gradient: detached, or an error."""
    _no_gradient(W_U=W_U, advantage=advantage, old_logp=old_logp, ref_logp=ref_logp)
    return _Policy.apply(rows, W_U, ids, advantage, old_logp, weight, dict(ref_logp=ref_logp, clip=clip, kl=kl, temperature=temperature))


def preference(rows, W_U, ids, offsets, *, ref_logp=None, weight=None, beta=0.1, smoothing=0.0, form="logistic", mean=False, temperature=1.0):
    """ll_preference, differentiable in the rows and the weight: (weight times every pair's loss, the scores [pairs, 2], the tokens'
    log-probabilities), the last two without a gradient.  The rows' gradient is formed with the loss, as in `distill`: give the weights here, and
    sum.  W_U and ref_logp get no gradient: detached, or an error."""
    _no_gradient(W_U=W_U, ref_logp=ref_logp)
    return _Preference.apply(rows, W_U, ids, offsets, weight,
                             dict(ref_logp=ref_logp, beta=beta, smoothing=smoothing, form=form, mean=mean, temperature=temperature))


class AdamW(torch.optim.Optimizer):
    """ll_adamw as an optimiser: all parameters of a group in one call, fp32 or bf16 (which are rounded stochastically), on the GPU, contiguous.

    max_norm: the gradients of all groups together are clipped to it (ll_grad_norm), and a step whose norm is not finite changes no parameter
    and no state, though it counts as a step: nothing waits for the GPU.  The norm of the last step is `norm`, a tensor.  bits: 32, or 8 for states
    of one byte.  seed: of the stochastic rounding.  copies: {parameter: bf16 tensor}, which gets the parameter's new values with every step.  For a
    captured step there is ll_adamw itself with a clock: this class counts on the host, and says so instead of being captured.
    """

    STATES = ("m", "v", "m_scale", "v_scale")

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, *, max_norm=None, bits=32, seed=0, copies=None):
        if bits not in (8, 32):
            raise ValueError(f"bits: {bits}, expected 8 or 32")
        if max_norm is not None and not max_norm > 0:
            raise ValueError(f"max_norm: {max_norm}, expected a positive number or None")
        self.max_norm, self.bits, self.seed, self.norm = max_norm, bits, seed, None
        self.copies = {} if copies is None else dict(copies)
        self._lists = {}
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))

    def _state(self, p):
        s = self.state[p]
        if not s:
            zeros = lambda dtype, n=None: torch.zeros(p.shape if n is None else (n,), dtype=dtype, device=p.device)
            blocks = -(-p.numel() // LL.LL_STATE_BLOCK)
            s["step"] = 0
            if self.bits == 32:
                s["m"], s["v"] = zeros(torch.float32), zeros(torch.float32)
            else:
                s["m"], s["v"] = zeros(torch.uint8).view(torch.float8_e4m3fn), zeros(torch.uint8).view(torch.float8_e5m2)
                s["m_scale"], s["v_scale"] = zeros(torch.float32, blocks), zeros(torch.float32, blocks)
        return s

    def _list(self, key, params, states, grads):
        """The parameters' TensorList, kept from step to step, with this step's gradients (which it lets go with the step)."""
        copies = [self.copies.get(p) for p in params] if self.copies else [None] * len(params)
        # (the list keeps its tensors' memory: what begins where one of them does is that one, unless it has been given other memory)
        where = [(p.data_ptr(), p.dtype, [x.data_ptr() for x in map(s.get, self.STATES) if x is not None], None if c is None else c.data_ptr())
                 for p, s, c in zip(params, states, copies)]
        found = self._lists.get(key)
        if found is not None and found[0] == where:
            found[1].set_grads(grads)
            return found[1]
        kept = LL.TensorList(grads, params, *([s.get(name) for s in states] for name in self.STATES), copies)
        self._lists[key] = where, kept
        return kept

    @staticmethod
    def _whole(g):
        """A gradient as the library takes it: dense, contiguous, from a multiple of 16 bytes on."""
        if g.layout != torch.strided:
            raise ValueError(f"a gradient is {g.layout}: only dense ones")
        g = g.contiguous()
        return g if g.data_ptr() % 16 == 0 else g.clone()

    def __getstate__(self):
        return dict(super().__getstate__(), max_norm=self.max_norm, bits=self.bits, seed=self.seed, norm=None, copies=self.copies, _lists={})

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        if torch.cuda.is_available() and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("a captured step would repeat one step number: capture ll_adamw with a clock")
        try:
            self._step()
        finally:
            # (kept, this step's gradients would stand in memory beside those of the next backward pass)
            for _, tensors in self._lists.values():
                tensors.set_grads([None] * len(tensors))
        return loss

    def _step(self):
        calls, used = [], set()
        for at, group in enumerate(self.param_groups):
            by_step = {}                                  # (parameters that were without a gradient at times have done fewer steps)
            for p in group["params"]:
                if p.grad is not None:
                    state = self._state(p)
                    params, states, grads = by_step.setdefault(state["step"], ([], [], []))
                    params.append(p)
                    states.append(state)
                    grads.append(self._whole(p.grad))
            for turn, (done, (params, states, grads)) in enumerate(by_step.items()):
                used.add((at, turn))
                calls.append((group, done + 1, params, states, self._list((at, turn), params, states, grads)))
        # (a group whose parameters are at one step again needs one list; one that had no gradients keeps its own)
        if len(self._lists) > len(used):
            self._lists = {key: kept for key, kept in self._lists.items() if key in used or (key[0], 0) not in used}
        if not calls:
            return
        self.norm = None
        if self.max_norm is not None:
            one = calls[0][-1] if len(calls) == 1 else LL.TensorList([g for *_, tensors in calls for g in tensors.grads])
            self.norm = LL.ll_grad_norm(one)
        for turn, (group, step, params, states, tensors) in enumerate(calls):
            LL.ll_adamw(tensors, step, rate=float(group["lr"]), betas=group["betas"], eps=group["eps"], decay=group["weight_decay"], norm=self.norm,
                        max_norm=float("inf") if self.max_norm is None else self.max_norm, seed=self.seed + turn)
            for state in states:
                state["step"] = step
            torch.autograd.graph.increment_version(params + [c for c in map(self.copies.get, params) if c is not None] if self.copies else params)

    def load_state_dict(self, state_dict):
        """As torch's, which would bring every state to its parameter's type: here they keep their own.  Hooks before it may give other states, and hooks
        behind it see those that were loaded."""
        given = []
        ours = [self.register_load_state_dict_pre_hook(lambda _, state_dict: given.append(state_dict)),
                self.register_load_state_dict_post_hook(lambda _: self._take(given[-1]), prepend=True)]
        try:
            super().load_state_dict(state_dict)
        finally:
            for hook in ours:
                hook.remove()

    def _take(self, state_dict):
        theirs = [i for group in state_dict["param_groups"] for i in group["params"]]
        ours = [p for group in self.param_groups for p in group["params"]]
        for i, p in zip(theirs, ours):
            if i in state_dict["state"]:
                self.state[p] = {k: x.detach().clone().to(p.device) if isinstance(x, torch.Tensor) else x for k, x in state_dict["state"][i].items()}
        self._lists = {}


class Translator(torch.nn.Module):
    """x = h + scale gate (h A^T + b), then the model's own final norm.  A and b start at zero: the raw lens.  Master weights are fp32, the
    products bf16."""

    def __init__(self, d: int, gamma: torch.Tensor, eps: float, scale: float = 1.0):
        super().__init__()
        like = {"dtype": torch.float32, "device": gamma.device}
        self.A = torch.nn.Parameter(torch.zeros((d, d), **like))
        self.b = torch.nn.Parameter(torch.zeros((d,), **like))
        self.gate = torch.nn.Parameter(torch.ones((d,), **like))
        self.register_buffer("gamma", gamma)
        self.eps, self.scale = eps, scale

    def forward(self, hidden):
        bf16 = torch.bfloat16
        y = torch.nn.functional.linear(hidden, self.A.to(bf16), self.b.to(bf16))
        return block_norm(hidden, y, self.gamma, self.eps, gate=self.gate, scale=self.scale)[1]


def teacher_of(last_hidden, gamma, W_U, eps, k):
    """The last layer's k most likely tokens and their log-probabilities, as ll_distill takes them."""
    ids, p, _, _ = LL.ll_project(last_hidden, gamma, W_U, eps, k)
    return ids, p.log()


@dataclass
class Fit:
    losses: list            # mean loss of every step
    logp_before: float      # mean log-probability of the teacher's first token, by the raw lens
    logp_after: float       # and by the translator


def fit(translator, hidden, last_hidden, W_U, *, k=20, temperature=1.0, steps=200, rate=1e-3, optimiser=None):
    """Trains a translator on one layer's rows against the last layer's read-out of the same tokens; optimiser: as made of its parameters,
    None: torch's Adam."""
    N, W_U = hidden.shape[0], W_U.detach()      # (the model's own: not trained)
    ids, scores = teacher_of(last_hidden, translator.gamma, W_U, translator.eps, k)
    weight = torch.full((N,), 1.0 / N, dtype=torch.float32, device=hidden.device)
    first = lambda: float(token_logp(translator(hidden), W_U, ids[:, :1].contiguous())[0].mean())
    with torch.no_grad():
        before = first()
    optimiser = torch.optim.Adam(translator.parameters(), lr=rate) if optimiser is None else optimiser(translator.parameters())
    losses = []
    for _ in range(steps):
        optimiser.zero_grad(set_to_none=True)
        loss = distill(translator(hidden), W_U, ids, scores, temperature=temperature, weight=weight).sum()
        loss.backward()
        optimiser.step()
        losses.append(loss.detach())
    with torch.no_grad():
        after = first()
    return Fit([float(x) for x in losses], before, after)


def fit_policy(translator, hidden, W_U, ids, advantage, *, updates=8, rate=1e-3, clip=(0.2, 0.2), kl=0.0, temperature=1.0, bits=32, max_norm=1.0):
    """Some updates on one sample of tokens and their advantages: ids and advantage, one a row (an id outside the vocabulary: none).  The sampling
    policy, and the reference of the KL term, is the translator as it comes.  Returns every update's mean loss."""
    W_U = W_U.detach()
    weight = (ids.reshape(-1) >= 0) & (ids.reshape(-1) < W_U.shape[0])
    weight = weight.float() / weight.sum().clamp(min=1)
    with torch.no_grad():
        _, old, _ = LL.ll_policy(translator(hidden), W_U, ids, advantage, temperature=temperature, grad=False)
    old = torch.nan_to_num(old)                           # (of rows without a token)
    optimiser, losses = AdamW(translator.parameters(), lr=rate, weight_decay=0.0, bits=bits, max_norm=max_norm), []
    for _ in range(updates):
        optimiser.zero_grad(set_to_none=True)
        loss, _ = policy(translator(hidden), W_U, ids, advantage, old, ref_logp=old, weight=weight, clip=clip, kl=kl, temperature=temperature)
        loss.sum().backward()
        optimiser.step()
        losses.append(loss.detach().sum())
    return [float(x) for x in losses]


@dataclass
class Preferred:
    losses: list             # mean loss of every step
    scores: torch.Tensor     # [pairs, 2] after the last: how much likelier than before each answer is


def fit_preference(translator, hidden, W_U, ids, offsets, *, steps=50, rate=1e-3, beta=0.1, smoothing=0.0, form="logistic", mean=False, bits=32,
                   max_norm=1.0):
    """Trains a translator to tell pairs of answers apart: ids one a row, offsets as ll_preference takes them.  The reference is the translator as it
    comes."""
    W_U, P = W_U.detach(), offsets.shape[0] // 2
    weight = torch.full((P,), 1.0 / P, dtype=torch.float32, device=hidden.device)
    options = dict(beta=beta, smoothing=smoothing, form=form, mean=mean)
    with torch.no_grad():
        ref = torch.nan_to_num(preference(translator(hidden), W_U, ids, offsets, **options)[2])
    optimiser, losses = AdamW(translator.parameters(), lr=rate, weight_decay=0.0, bits=bits, max_norm=max_norm), []
    for _ in range(steps):
        optimiser.zero_grad(set_to_none=True)
        loss, _, _ = preference(translator(hidden), W_U, ids, offsets, ref_logp=ref, weight=weight, **options)
        loss.sum().backward()
        optimiser.step()
        losses.append(loss.detach().sum())
    with torch.no_grad():
        _, score, _ = preference(translator(hidden), W_U, ids, offsets, ref_logp=ref, **options)
    return Preferred([float(x) for x in losses], score)


def synthetic_layers(N, d, V, device, seed=0):
    """An inner layer's rows and the last layer's of the same tokens, which are a fixed map of them and some noise; gamma and W_U."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device=device)
    inner = normal(N, d)
    last = inner + 0.7 * inner @ normal(d, d) / d ** 0.5 + 0.1 * normal(N, d)
    W_U = (4.0 * normal(V, d) / d ** 0.5).to(torch.bfloat16)
    return inner.to(torch.bfloat16), last.to(torch.bfloat16), torch.ones((d,), dtype=torch.bfloat16, device=device), W_U


def main():
    inner, last, gamma, W_U = synthetic_layers(2048, 256, 4096, "cuda:0")
    result = fit(Translator(256, gamma, 1e-5), inner, last, W_U)
    print(f"distillation loss {result.losses[0]:.3f} -> {result.losses[-1]:.3f}; the last layer's token, log-probability "
          f"{result.logp_before:.3f} -> {result.logp_after:.3f}")
    # 64 pairs of 16-token answers over the same rows: the last layer's own tokens are preferred to any others
    ids = LL.ll_project(last, gamma, W_U, 1e-5, 1)[0].reshape(64, 2, 16)
    ids[:, 1] = torch.randint(0, 4096, (64, 16), dtype=torch.int32, device=ids.device)
    offsets = torch.arange(0, 2049, 16, dtype=torch.int32, device=ids.device)
    preferred = fit_preference(Translator(256, gamma, 1e-5), inner, W_U, ids.reshape(-1), offsets, bits=8)
    print(f"preference loss {preferred.losses[0]:.3f} -> {preferred.losses[-1]:.3f}, the preferred answer ahead in "
          f"{int((preferred.scores[:, 0] > preferred.scores[:, 1]).sum())} of 64")


if __name__ == "__main__":
    main()
