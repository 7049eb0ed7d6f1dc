"""The fp64 oracle of what learns from answers against central differences and known values (no GPU needed)."""
import numpy as np
import pytest

import oracle.answers_oracle as O


def small(seed=0, N=7, d=6, V=11):
    g = np.random.default_rng(seed)
    rows, W = g.normal(size=(N, d)), g.normal(size=(V, d))
    ids = g.integers(0, V, N)
    ids[3] = -1
    return g, rows, W, ids


def differences(f, rows, h=1e-6):
    out = np.zeros_like(rows)
    for i in np.ndindex(rows.shape):
        a, b = rows.copy(), rows.copy()
        a[i] += h
        b[i] -= h
        out[i] = (f(a) - f(b)) / (2 * h)
    return out


@pytest.mark.parametrize("kl,low,high", [(0.0, 0.2, 0.2), (0.3, 0.15, 0.4), (0.2, 1.0, np.inf)])     # (no ratio on a border, where there is no derivative)
def test_policy(kl, low, high):
    g, rows, W, ids = small()
    A, weight = g.normal(size=7), g.random(7)
    at = O.policy(rows, W, ids, A, temperature=0.7)[1]
    old, ref = np.where(ids >= 0, at, 0.0) - np.log([0.7, 0.9, 1.5, 1.0, 1.1, 0.5, 1.3]), np.where(ids >= 0, at, 0.0) + 0.4 * g.normal(size=7)
    f = lambda x: float(np.sum(weight * O.policy(x, W, ids, A, old, ref, weight, low, high, kl, 0.7)[0]))
    loss, logp, dz, size = O.policy(rows, W, ids, A, old, ref, weight, low, high, kl, 0.7)
    assert np.allclose(dz @ W, differences(f, rows), atol=1e-8) and np.all(size >= np.abs(dz) - 1e-15)
    assert loss[3] == 0 and np.isnan(logp[3]) and not dz[3].any()


def test_policy_of_its_own_samples():
    """On policy the ratio is 1: the loss is -A, its gradient that of -A l."""
    g, rows, W, ids = small(1)
    A = g.normal(size=7)
    loss, logp, dz, _ = O.policy(rows, W, ids, A)
    assert np.allclose(loss, np.where(ids >= 0, -A, 0))
    f = lambda x: float(np.nansum(-A * O.policy(x, W, ids, A)[1]))
    assert np.allclose(dz @ W, differences(f, rows), atol=1e-8)


@pytest.mark.parametrize("form", ["logistic", "hinge", "square"])
@pytest.mark.parametrize("mean", [False, True])
def test_preference(form, mean):
    g, rows, W, ids = small(2)
    offsets, ref, weight = np.array([0, 2, 4, 4, 6]), g.normal(size=7) - 2, np.array([0.6, 1.7])
    kw = dict(ref=ref, weight=weight, beta=0.3, smoothing=0.1 if form == "logistic" else 0.0, form=form, mean=mean)
    f = lambda x: float(np.sum(weight * O.preference(x, W, ids, offsets, **kw)[0]))
    loss, score, logp, dz, _ = O.preference(rows, W, ids, offsets, **kw)
    assert np.allclose(dz @ W, differences(f, rows), atol=1e-7)
    assert score[1, 0] == 0 and not dz[3].any() and not dz[6].any()
    assert np.isclose(score[0, 1], logp[2] - ref[2])            # row 3 holds no token


def test_logistic_at_zero_and_far_out():
    assert np.isclose(O.pair_loss("logistic", 0.0, 1.0)[0], np.log(2)) and O.pair_loss("logistic", 0.0, 1.0)[1] == -0.5
    loss, slope = O.pair_loss("logistic", -800.0, 1.0)
    assert loss == 800 and slope == -1
