"""What learns through the lens, in fp64: the norms around a block, log-probabilities of listed tokens, distillation from a teacher's
top tokens, and the gradient of each.  Written from the definitions; NumPy only.
"""
import numpy as np


def _rms(x, eps):
    return np.sqrt(np.mean(x * x, axis=1, keepdims=True) + eps)


def block_norm(h, y, gamma, eps, gate=None, scale=1.0, gamma_y=None):
    """(x, gamma x / rms(x)) with x = h + scale gate u, u = y or gamma_y y / rms(y)."""
    u = y if gamma_y is None else gamma_y * y / _rms(y, eps)
    x = h + scale * (1.0 if gate is None else gate) * u
    return x, gamma * x / _rms(x, eps)


def block_norm_grad(h, y, gamma, eps, g_hidden, g_normed, gate=None, scale=1.0, gamma_y=None):
    """The gradients (d_h, d_y, d_gate of every row, d_gamma_y, d_gamma), and beside each the sum of the sizes of what it is made of,
    which is what rounding errors scale with."""
    d = h.shape[1]
    r_y = _rms(y, eps)
    yh = y / r_y
    u = y if gamma_y is None else gamma_y * yh
    k = scale * (np.ones_like(h) if gate is None else gate * np.ones_like(h))
    x = h + k * u
    size_x = np.abs(h) + np.abs(k * u)
    r = _rms(x, eps)
    xh, size_xh = x / r, size_x / r
    e = g_normed * gamma
    dx = g_hidden + (e - xh * np.mean(e * xh, axis=1, keepdims=True)) / r
    size_dx = np.abs(g_hidden) + (np.abs(e) + size_xh * np.mean(np.abs(e) * size_xh, axis=1, keepdims=True)) / r
    du, size_du = k * dx, np.abs(k) * size_dx
    d_gate, size_gate = scale * u * dx, np.abs(scale * u) * size_dx
    d_gamma, size_gamma = np.sum(g_normed * xh, axis=0), np.sum(np.abs(g_normed) * size_xh, axis=0)
    if gamma_y is None:
        return (dx, du, d_gate, None, d_gamma), (size_dx, size_du, size_gate, None, size_gamma)
    f, size_f = du * gamma_y, size_du * np.abs(gamma_y)
    dy = (f - yh * np.mean(f * yh, axis=1, keepdims=True)) / r_y
    size_dy = (size_f + np.abs(yh) * np.mean(size_f * np.abs(yh), axis=1, keepdims=True)) / r_y
    return ((dx, dy, d_gate, np.sum(du * yh, axis=0), d_gamma),
            (size_dx, size_dy, size_gate, np.sum(size_du * np.abs(yh), axis=0), size_gamma))


def _log_softmax(rows, W, temperature):
    z = rows @ W.T / temperature
    m = np.max(z, axis=1, keepdims=True)
    lse = m + np.log(np.sum(np.exp(z - m), axis=1, keepdims=True))
    return z - lse, lse[:, 0]


def logp(rows, W, ids, temperature=1.0):
    """(logp [N, k], NaN for an id outside the vocabulary, logsumexp [N], entropy [N])"""
    lp, lse = _log_softmax(rows, W, temperature)
    V = W.shape[0]
    ok = (ids >= 0) & (ids < V)
    listed = np.take_along_axis(lp, np.where(ok, ids, 0), axis=1)
    return np.where(ok, listed, np.nan), lse, -np.sum(np.exp(lp) * lp, axis=1)


def logp_grad(rows, W, ids, g_logp, g_entropy=None, temperature=1.0):
    """dz [N, V], d / d logits of sum g_logp logp + sum g_entropy entropy, before its product with W, and the size of its parts."""
    lp, _ = _log_softmax(rows, W, temperature)
    p, V = np.exp(lp), W.shape[0]
    dz, size = np.zeros_like(lp), np.zeros_like(lp)
    for r in range(rows.shape[0]):
        for i, v in enumerate(ids[r]):
            if 0 <= v < V:
                g = g_logp[r, i]
                dz[r] -= g * p[r]
                dz[r, v] += g
                size[r] += abs(g) * p[r]
                size[r, v] += abs(g)
    if g_entropy is not None:
        H = -np.sum(p * lp, axis=1, keepdims=True)
        dz -= g_entropy[:, None] * p * (lp + H)
        size += np.abs(g_entropy[:, None]) * p * (np.abs(lp) + H)
    return dz / temperature, size / temperature


def distill(rows, W, ids, scores, temperature=1.0, weight=None):
    """(loss [N], dz [N, V], the size of its parts)"""
    lp, _ = _log_softmax(rows, W, temperature)
    V, N = W.shape[0], rows.shape[0]
    loss, dz, size = np.zeros(N), np.zeros_like(lp), np.zeros_like(lp)
    for r in range(N):
        entries = [i for i, v in enumerate(ids[r]) if 0 <= v < V and scores[r, i] != -np.inf]
        if not entries:
            continue
        s = scores[r, entries] / temperature
        log_t = s - np.max(s)
        log_t = log_t - np.log(np.sum(np.exp(log_t)))
        t, at = np.exp(log_t), ids[r, entries]
        loss[r] = temperature ** 2 * np.sum(t * (log_t - lp[r, at]))
        w = 1.0 if weight is None else weight[r]
        if w == 0.0:
            continue
        dz[r] = np.exp(lp[r])
        size[r] = dz[r]
        np.subtract.at(dz[r], at, t)
        np.add.at(size[r], at, t)
        dz[r] *= temperature * w
        size[r] *= abs(temperature * w)
    return loss, dz, size
