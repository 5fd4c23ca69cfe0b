"""The token losses' 64-bit oracle: known values, and gradients against differences of
the losses."""
import numpy as np
import pytest

from oracle import token_loss as tl


def data(n=9, V=13, seed=0, masked=False):
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(n, V)) * 2
    tok = rng.integers(0, V, n)
    if masked:
        z[rng.random((n, V)) < 0.3] = -np.inf
        z[np.arange(n), tok] = 1.0
    tok[2] = -1
    return rng, z, tok


def differences(f, z, h=1e-5):
    """Central differences of f at the finite entries of z."""
    g = np.zeros_like(z)
    for i in np.ndindex(z.shape):
        if np.isfinite(z[i]):
            up, dn = z.copy(), z.copy()
            up[i] += h
            dn[i] -= h
            g[i] = (f(up) - f(dn)) / (2 * h)
    return g


# a central difference is off by h^2 / 6 of the third derivative (of order 1) and 2^-52 / h of the value
TOL = dict(rtol=1e-7, atol=1e-9)


def test_uniform_rows():
    lp, p, H, live = tl.rows(np.full((2, 8), -3e38), 0.5)
    np.testing.assert_allclose(lp, -np.log(8))
    np.testing.assert_allclose(p, 1 / 8)
    np.testing.assert_allclose(H, np.log(8))
    assert live.all()
    assert not tl.rows(np.full((1, 4), -np.inf))[3].any()


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("T", [1.0, 0.6, 2.0])
def test_ppo_gradient(T, masked):
    rng, z, tok = data(masked=masked)
    n = len(tok)
    logp = tl.logprob(z, tok, T)[0]
    old = logp - rng.choice([-0.5, -0.1, 0.1, 0.5], n)          # both clip sides and the middle
    adv, ref, w = rng.normal(size=n), logp + rng.normal(size=n) * 0.3, rng.random(n)
    args = (tok, old, adv, w, ref, 0.2, 0.3, 0.7, 0.11, T)
    g = tl.ppo(z, *args)[1]
    np.testing.assert_allclose(g, differences(lambda x: tl.ppo(x, *args)[0], z), **TOL)
    assert not g[2].any()


@pytest.mark.parametrize("T", [1.0, 1.7])
def test_pref_gradient(T):
    rng, z, tok = data(n=11, seed=1)
    off = np.array([0, 3, 3, 5, 11])                             # an empty answer too
    args = (tok, off, rng.normal(size=11) - 2, 0.4, 0.1, T)
    np.testing.assert_allclose(tl.pref(z, *args)[1], differences(lambda x: tl.pref(x, *args)[0], z), **TOL)


@pytest.mark.parametrize("T", [1.0, 2.0])
def test_distill_gradient(T):
    rng, z, tok = data(n=7, seed=2)
    ids = rng.integers(0, 13, (7, 5))                            # some twice
    ids[1, 2:], ids[4] = -1, -1
    t = rng.normal(size=(7, 5)) * 3
    t[0, 1] = -np.inf
    args = (ids, t, rng.random(7), T)
    g = tl.distill(z, *args)[1]
    np.testing.assert_allclose(g, differences(lambda x: tl.distill(x, *args)[0], z), **TOL)
    assert not g[4].any()


def test_distill_from_itself_is_a_minimum():
    _, z, _ = data(n=3, seed=3)
    ids = np.tile(np.arange(13), (3, 1))
    L, g, loss, q, _ = tl.distill(z, ids, z, np.ones(3), 1.5)
    np.testing.assert_allclose(loss, 0, atol=1e-14)
    np.testing.assert_allclose(g, 0, atol=1e-15)


def test_pref_of_equal_answers():
    _, z, tok = data(n=4, seed=4)
    z[2:], tok[:] = z[:2], [3, 4, 3, 4]
    L, g, R, _, stats = tl.pref(z, tok, np.array([0, 2, 4]), None, 0.5)
    assert abs(L - np.log(2)) < 1e-15 and R[0] == R[1] and stats[2] == 0
    np.testing.assert_allclose(g[:2], -g[2:])
