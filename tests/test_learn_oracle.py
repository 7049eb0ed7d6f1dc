"""The oracle's gradients against central differences of its own forward values (no GPU needed)."""
import numpy as np
import pytest

import oracle.learn_oracle as O

STEP = 1e-5
# central differences in fp64: third derivatives of O(10) times STEP^2 / 6, and 2^-52 |f| / STEP of rounding, both below 1e-8 here
TOL = 1e-7


def numeric(f, x):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        keep = x[i]
        x[i] = keep + STEP
        up = f()
        x[i] = keep - STEP
        down = f()
        x[i] = keep
        g[i] = (up - down) / (2 * STEP)
    return g


@pytest.mark.parametrize("gate_kind", ["none", "shared", "rows"])
@pytest.mark.parametrize("post", [False, True])
def test_block_norm(gate_kind, post):
    rng = np.random.default_rng(7)
    N, d, eps, scale = 3, 8, 1e-3, 0.7
    h, y, gx, gn = (rng.standard_normal((N, d)) for _ in range(4))
    gamma, gamma_y = 1 + 0.1 * rng.standard_normal(d), 1 + 0.1 * rng.standard_normal(d) if post else None
    gate = {"none": None, "shared": rng.standard_normal(d), "rows": rng.standard_normal((N, d))}[gate_kind]

    def value():
        x, n = O.block_norm(h, y, gamma, eps, gate, scale, gamma_y)
        return np.sum(x * gx) + np.sum(n * gn)

    (dh, dy, dk, dgy, dg), sizes = O.block_norm_grad(h, y, gamma, eps, gx, gn, gate, scale, gamma_y)
    pairs = [(dh, h), (dy, y), (dg, gamma)]
    if gate is not None:
        pairs.append((dk.sum(0) if gate_kind == "shared" else dk, gate))
    if post:
        pairs.append((dgy, gamma_y))
    for got, at in pairs:
        np.testing.assert_allclose(got, numeric(value, at), atol=TOL, rtol=TOL)
    for g, s in zip((dh, dy, dk, dgy, dg), sizes):
        assert g is None or np.all(np.abs(g) <= s * (1 + 1e-12))


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_logp(temperature):
    rng = np.random.default_rng(8)
    N, d, V, k = 3, 6, 9, 4
    rows, W = rng.standard_normal((N, d)), rng.standard_normal((V, d))
    ids = rng.integers(0, V, (N, k))
    ids[0, 1] = ids[0, 0]                   # one token twice
    ids[1, 2], ids[2, :] = -1, V            # entries, and a row, that take no part
    g, gh = rng.standard_normal((N, k)), rng.standard_normal(N)

    def value():
        lp, _, ent = O.logp(rows, W, ids, temperature)
        return np.nansum(lp * g) + np.sum(ent * gh)

    dz, size = O.logp_grad(rows, W, ids, g, gh, temperature)
    np.testing.assert_allclose(dz @ W, numeric(value, rows), atol=TOL, rtol=TOL)
    assert np.all(np.abs(dz) <= size * (1 + 1e-12))


@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_distill(temperature):
    rng = np.random.default_rng(9)
    N, d, V, k = 4, 6, 9, 4
    rows, W = rng.standard_normal((N, d)), rng.standard_normal((V, d))
    ids, scores, weight = rng.integers(0, V, (N, k)), rng.standard_normal((N, k)), rng.random(N)
    ids[0, 1], ids[1, 2], ids[2, :], scores[3, 0] = ids[0, 0], V + 3, -1, -np.inf

    def value():
        return np.sum(weight * O.distill(rows, W, ids, scores, temperature)[0])

    loss, dz, size = O.distill(rows, W, ids, scores, temperature, weight)
    assert loss[2] == 0 and not dz[2].any()
    np.testing.assert_allclose(dz @ W, numeric(value, rows), atol=TOL, rtol=TOL)
    assert np.all(np.abs(dz) <= size * (1 + 1e-12))
    # a teacher that is the student itself costs nothing and teaches nothing
    lp = O.logp(rows, W, np.tile(np.arange(V), (N, 1)), temperature)[0]
    loss, dz, _ = O.distill(rows, W, np.tile(np.arange(V), (N, 1)), lp * temperature, temperature)
    np.testing.assert_allclose(loss, 0, atol=1e-12)
    np.testing.assert_allclose(dz, 0, atol=1e-12)
