"""The gradient of a log decay: e^g_t <S_{t-1}, dS'_t>, as small as the decay makes it.  Two ways to have it from a chunk's inner values in 32 bits, and
that the bound (oracle.delta.delta_bounds, dg_divided) tells one from the other."""
import numpy as np
import pytest

from oracle import delta as R

f = np.float32


def _terms(q, k, v, g, beta, dO, S, dS):
    """One chunk in 64 bits: X o (q . k) - beta Y o (k . k) of all pairs (in front on the diagonal too), what a token has from the state, what it hands on,
    and what goes through."""
    n = len(k)
    gamma = np.cumsum(np.maximum(g, -256.0))
    D = np.tril(np.exp(np.tril(gamma[:, None] - gamma[None])))
    up, down, whole = np.exp(gamma)[:, None], np.exp(gamma[-1] - gamma)[:, None], np.exp(gamma[-1])
    be = beta[:, None]
    T = np.linalg.inv(np.eye(n) + np.tril(be * D * (k @ k.T), -1))
    U = T @ (be * (v - up * (k @ S)))
    dR = T.T @ ((D * (q @ k.T)).T @ dO + down * (k @ dS))
    X, Y = D * (dO @ U.T), np.tril(D, -1) * (dR @ U.T)
    W = X * (q @ k.T) - be * Y * (k @ k.T)
    near = (q * (up * (dO @ S.T))).sum(1) - (k * (be * up * (dR @ S.T))).sum(1)
    return W, near, (k * (down * (U @ dS.T))).sum(1), whole * (S * dS).sum()


def _differences_of_sums(W, near, far, through):
    """dgamma of every token, then its suffix sums: pairs on one side of t cancel."""
    d = (W.sum(1, dtype=f) + near) - (W.sum(0, dtype=f) + far)
    d[-1] += through + far.sum(dtype=f)
    return np.cumsum(d[::-1], dtype=f)[::-1]


def _divided(W, near, far, through):
    n = len(near)
    return np.array([W[t:, :t].sum(dtype=f) + near[t:].sum(dtype=f) + far[:t].sum(dtype=f) + through for t in range(n)], f)


def _inputs(rng, n, d, weak):
    def unit(x):
        return x / np.linalg.norm(x, axis=1, keepdims=True)
    g = -np.exp(rng.normal(size=n) - weak)
    return unit(rng.normal(size=(n, d))), unit(rng.normal(size=(n, d))), rng.normal(size=(n, d)), g, 1 / (1 + np.exp(-rng.normal(size=n)))


@pytest.mark.parametrize("weak", [-2.0, 0.0, 3.0])
def test_divided_pairs_are_the_gradient_and_keep_its_digits(rng, weak):
    n, d = 64, 64
    q, k, v, g, beta = _inputs(rng, n, d, weak)
    g[10], g[30] = -np.inf, -300.0
    dO, S, dS = rng.normal(size=(n, d)), 0.3 * rng.normal(size=(d, d)), 0.3 * rng.normal(size=(d, d))
    ref = R.delta_bwd(q, k, v, g, beta, dO, 1.0, S, dS)["dg"]
    bound = R.delta_bounds(q, k, v, g, beta, dO, n, 0.0, 0.0, 1.0, S, dS)["dg_divided"]
    t64 = _terms(q, k, v, g, beta, dO, S, dS)
    assert np.allclose(_divided(*t64), ref, rtol=1e-5, atol=1e-6 * np.abs(ref).max())
    t32 = [np.asarray(x, f) for x in t64]
    off = np.abs(_divided(*t32) - ref)
    assert (off <= bound + 2.0 ** -24 * np.abs(ref) + 2.0 ** -126).all()
    assert max(bound[10], bound[30], abs(ref[10]), abs(ref[30])) <= 1e-100            # (the bound holds log decays to -256)
    if weak < 0:
        # the other way many tokens have no digit left, though the head as a whole looks right
        other = _differences_of_sums(*t32)
        assert np.linalg.norm(other - ref) <= 1e-4 * np.linalg.norm(ref)
        assert (np.abs(other - ref) > bound + 2.0 ** -24 * np.abs(ref)).sum() >= 3
        assert other[10] != 0 or other[30] != 0
    assert (bound <= 1e-2 * np.abs(ref) + 1e-30).mean() >= 0.5


def test_the_bound_has_the_decay_of_each_token(rng):
    q, k, v, g, beta = _inputs(rng, 100, 64, 2.0)
    dO = rng.normal(size=(100, 64))
    args = lambda g: (q, k, v, g, beta, dO, 64, 2.0 ** -8, 2.0 ** -16)  # noqa: E731
    a = R.delta_bounds(*args(g))["dg_divided"]
    h = g.copy()
    h[50] -= 20
    b = R.delta_bounds(*args(h))["dg_divided"]
    assert b[50] <= 2 * np.exp(-20) * a[50] and a[0] == 0
