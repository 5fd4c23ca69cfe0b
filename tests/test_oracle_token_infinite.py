"""The token losses' 64-bit oracle where a factor is infinite or overflows."""
import numpy as np

from oracle import token_loss as tl

Z = np.array([[0.5, -1.0, 2.0, -np.inf], [1.0, 0.0, -0.5, 0.25]])
TOK = np.array([2, 1])
W = np.array([0.5, 0.5])


def test_reference_with_coefficient_zero():
    lp = tl.logprob(Z, TOK)[0]
    plain = tl.ppo(Z, TOK, lp, np.ones(2), W)
    L, g, _, _, _, stats = tl.ppo(Z, TOK, lp, np.ones(2), W, ref=lp + [800.0, 0.1])
    assert L == plain[0] and np.array_equal(g, plain[1]) and stats[3] == np.inf


def test_ratio_past_the_type_with_advantage_zero():
    lp = tl.logprob(Z, TOK)[0]
    want = tl.ppo(Z, TOK, lp, np.array([0.0, 1.0]), W, ch=0.1)
    got = tl.ppo(Z, TOK, lp - [800.0, 0.0], np.array([0.0, 1.0]), W, ch=0.1)
    assert got[0] == want[0] and np.array_equal(got[1], want[1])


def test_kl_of_a_masked_token():
    tok = np.array([3, 1])
    L, _, logp, l, _, stats = tl.ppo(Z, tok, np.array([-1.0, -1.0]), np.ones(2), W, ref=np.array([-1.0, -1.0]), ck=0.1)
    assert logp[0] == -np.inf and l[0] == L == stats[3] == np.inf and np.isfinite(l[1])


def test_gradient_of_an_infinite_slope():
    """Masked entries stay 0, the others go to the infinity of their sign."""
    tok = np.array([0, 1])
    z = np.array([[-np.inf, -1.0, 2.0, -np.inf], [1.0, 0.0, -0.5, 0.25]])
    for ref in ([-1.0, -1.0], [-1.0, 900.0]):
        g = tl.ppo(z, tok, np.array([-1.0, -1.0]), np.ones(2), W, ref=np.array(ref), ck=0.1)[1]
        assert np.array_equal(g[0], [-np.inf, np.inf, np.inf, 0])
        assert np.isfinite(g[1]).all() if ref[1] < 0 else np.array_equal(g[1], np.inf * np.array([1, -1, 1, 1]))


def test_pair_with_a_masked_rejected_token():
    z, off = np.vstack([Z[1], Z[0], Z[1], Z[1]]), np.arange(5)
    tok = np.array([1, 3, 0, 2])
    L, g, R, _, _ = tl.pref(z, tok, off, None, 0.5)
    assert R[1] == -np.inf and not g[:2].any() and L == np.logaddexp(0, -(R[2] - R[3])) / 2
    assert tl.pref(z, tok, off, None, 0.5, 0.1)[0] == np.inf
