"""What learns from answers, in fp64: a clipped policy loss with a KL term, a preference loss over pairs, AdamW and its states in 8 bits.
Written from the definitions; NumPy only.
"""
import numpy as np

from .learn_oracle import _log_softmax


def _rows_gradient(lp, ids, ok, c, temperature):
    """dz [N, V] of sum c l, and the size of its parts."""
    p = np.exp(lp)
    at = np.where(ok, ids, 0)[:, None]
    dz, size = -c[:, None] * p, np.abs(c)[:, None] * p
    np.put_along_axis(dz, at, np.take_along_axis(dz, at, 1) + c[:, None], 1)
    np.put_along_axis(size, at, np.take_along_axis(size, at, 1) + np.abs(c)[:, None], 1)
    return dz / temperature, size / temperature


def policy_c(logp, advantage, old=None, ref=None, low=0.2, high=0.2, kl=0.0):
    """(loss, d loss / d logp) of every token."""
    ratio = np.ones_like(logp) if old is None else np.exp(logp - old)
    clipped = np.where(advantage > 0, ratio > 1 + high, ratio < 1 - low)
    held = np.where(advantage > 0, 1 + high, 1 - low) if np.isfinite(high) else np.where(advantage > 0, ratio, 1 - low)
    loss = -advantage * np.where(clipped, held, ratio)
    c = np.where(clipped, 0.0, -advantage * ratio)
    if kl:
        q = ref - logp
        loss, c = loss + kl * (np.expm1(q) - q), c - kl * np.expm1(q)
    return loss, c


def policy(rows, W, ids, advantage, old=None, ref=None, weight=None, low=0.2, high=0.2, kl=0.0, temperature=1.0):
    """(loss [N], logp [N], dz [N, V], the size of its parts)"""
    lp, _ = _log_softmax(rows, W, temperature)
    ok = (ids >= 0) & (ids < W.shape[0])
    l = np.take_along_axis(lp, np.where(ok, ids, 0)[:, None], 1)[:, 0]
    loss, c = policy_c(l, advantage, old, ref, low, high, kl)
    w = np.ones_like(l) if weight is None else weight
    c = np.where(ok & (w != 0), w * c, 0.0)
    return (np.where(ok, loss, 0.0), np.where(ok, l, np.nan)) + _rows_gradient(lp, ids, ok, c, temperature)


def pair_loss(form, h, beta, smoothing=0.0):
    """(loss, d loss / d h)"""
    if form == "logistic":
        up, down = np.logaddexp(0, h), np.logaddexp(0, -h)          # -log sigmoid(-h), -log sigmoid(h)
        return (1 - smoothing) * down + smoothing * up, smoothing * np.exp(-down) - (1 - smoothing) * np.exp(-up)
    if form == "hinge":
        return max(0.0, 1 - h), -1.0 if h < 1 else 0.0
    return ((h - 0.5) / beta) ** 2, 2 * (h - 0.5) / beta ** 2


def preference(rows, W, ids, offsets, ref=None, weight=None, beta=0.1, smoothing=0.0, form="logistic", mean=False, temperature=1.0):
    """(loss [P], score [P, 2], logp [N], dz [N, V], the size of its parts)"""
    lp, _ = _log_softmax(rows, W, temperature)
    ok = (ids >= 0) & (ids < W.shape[0])
    l = np.take_along_axis(lp, np.where(ok, ids, 0)[:, None], 1)[:, 0]
    gain = l if ref is None else l - ref
    P = len(offsets) // 2
    loss, score, c = np.zeros(P), np.zeros((P, 2)), np.zeros(len(ids))
    for j in range(P):
        parts = [np.arange(offsets[2 * j + s], offsets[2 * j + s + 1]) for s in (0, 1)]
        parts = [r[ok[r]] for r in parts]
        length = [max(1, len(r)) if mean else 1 for r in parts]
        score[j] = [np.sum(gain[r]) / n for r, n in zip(parts, length)]
        loss[j], slope = pair_loss(form, beta * (score[j, 0] - score[j, 1]), beta, smoothing)
        w = 1.0 if weight is None else weight[j]
        for r, n, sign in zip(parts, length, (1, -1)):
            c[r] = 0.0 if w == 0 else sign * w * slope * beta / n
    return (loss, score, np.where(ok, l, np.nan)) + _rows_gradient(lp, ids, ok, c, temperature)
