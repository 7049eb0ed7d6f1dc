"""Training through the lens: translators that bring an inner layer's states to what the last layer's lens reads out.

The raw logit lens (ll_project) applies the model's final norm and unembedding to states that were never meant for them.  A translator
per layer, x = h + scale gate (h A^T + b), learns what is missing from the model itself: its teacher is the last layer's own read-out,
the k most likely tokens that ll_project lists.  Nothing of the model changes.

`block_norm`, `token_logp` and `distill` are the library's calls with their gradients, for torch's autograd; `Translator` and `fit`
put them together:

    rows  -> product with A (torch) -> ll_block_norm -> ll_distill -> gradient of the normed rows -> ll_block_norm_grad -> A, b, gate

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


def _no_gradient(**tensors):
    """What the library has no gradient of is refused where autograd would be asked for one: without it a training step would miss a term."""
    if torch.is_grad_enabled():
        for name, t in tensors.items():
            if t.requires_grad:
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


def fit(translator, hidden, last_hidden, W_U, *, k=20, temperature=1.0, steps=200, rate=1e-3):
    """Trains a translator on one layer's rows against the last layer's read-out of the same tokens."""
    N, W_U = hidden.shape[0], W_U.detach()      # (the model's own: not trained)
    ids, scores = teacher_of(last_hidden, translator.gamma, W_U, translator.eps, k)
    weight = torch.full((N,), 1.0 / N, dtype=torch.float32, device=hidden.device)
    first = lambda: float(token_logp(translator(hidden), W_U, ids[:, :1].contiguous())[0].mean())
    with torch.no_grad():
        before = first()
    optimiser = torch.optim.Adam(translator.parameters(), lr=rate)
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


if __name__ == "__main__":
    main()
