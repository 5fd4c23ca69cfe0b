"""The token losses where a factor of the formulas is infinite or overflows fp32: a term whose
coefficient is 0 adds 0, an infinite value stays infinite and does not become NaN, and masked
entries keep gradient 0."""
import numpy as np
import pytest

from gpu_util import context
from oracle import token_loss as tl
from test_gpu_token_losses import HALF_ULP, TINY, Batch, cuda, empty

pytestmark = pytest.mark.gpu

# one length for each kernel: a thread a row, 8 lanes, a warp in registers, a warp through shared
# memory, the ring, the ring in clusters (few rows)
LENGTHS = [12, 40, 300, 5000, 40_000, 150_001]
TYPES = ["f32", "bf16", "f16"]


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


def rows(V, dt, seed, pad=0):
    """Four rows with masked entries, whose tokens are not; and their ln p."""
    b = Batch(4, V, dt, seed, masked=0.3, out=0.0, pad=pad)
    return b, tl.logprob(b.z, b.tok)[0]


def ppo(ctx, b, old, adv, g=None, **kw):
    logp, stats = empty(b.n), empty(5)
    kw = {k: cuda(np.asarray(v, np.float32)) if k == "ref_logp" and v is not None else v for k, v in kw.items()}
    ctx.learn_token_ppo(b.logits, cuda(b.tok), cuda(np.asarray(old, np.float32)), cuda(np.asarray(adv, np.float32)), g,
                        stats, logp_out=logp, **kw)
    ctx.sync()
    return logp.cpu().numpy(), stats.cpu().numpy()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", LENGTHS)
def test_reference_with_coefficient_zero(ctx, V, dt):
    """The KL reported alone: no bit of loss and gradient differs from the call without a
    reference, also where e^(ref - ln p) exceeds fp32."""
    b, lp = rows(V, dt, V)
    adv, old = [1, -1, 0.5, 2], lp + 0.1
    (_, plain), (_, with_ref) = b.grad(), b.grad()
    logp0, s0 = ppo(ctx, b, old, adv, plain, entropy_coef=0.01)
    logp1, s1 = ppo(ctx, b, old, adv, with_ref, entropy_coef=0.01, ref_logp=lp + [0.1, 100, -0.2, -100])
    assert np.isfinite(s0).all() and np.array_equal(logp0, logp1) and bool((plain == with_ref).all())
    assert np.array_equal(s0[[0, 1, 2, 4]], s1[[0, 1, 2, 4]]) and s1[3] == np.inf
    _, s2 = ppo(ctx, b, old, adv, with_ref, entropy_coef=0.01, ref_logp=lp + [0.1, 80, -0.2, -100])
    np.testing.assert_allclose(s2[3], np.exp(80) / 4, rtol=1e-4)                  # 80 is known to its rounding and ln p's error


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", LENGTHS)
def test_ratio_past_fp32_with_advantage_zero(ctx, V, dt):
    """rho A of an advantage 0 is 0 whatever the ratio: the row adds nothing, and the entropy term
    is as it is without the ratio."""
    b, lp = rows(V, dt, V + 1)
    (_, g), (_, near) = b.grad(), b.grad()
    far = lp - [100, 0.1, 200, -0.1]
    _, stats = ppo(ctx, b, far, [0, 1, -0.0, -1], g, entropy_coef=0.5)
    _, want = ppo(ctx, b, lp - [0, 0.1, 0, -0.1], [0, 1, -0.0, -1], near, entropy_coef=0.5)
    assert np.isfinite(stats).all() and np.array_equal(stats, want) and bool((g == near).all())
    # the clipped term of a positive advantage is finite too, the unclipped one of a negative is not
    _, stats = ppo(ctx, b, far, [1, 0, 1, 0], g)
    np.testing.assert_allclose(stats[1], -2 * 1.2 / 4, rtol=1e-6)
    assert not g.any()
    _, stats = ppo(ctx, b, far, [-1, 0, 0, 0], g)
    assert stats[1] == np.inf


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", LENGTHS)
def test_kl_of_a_masked_token(ctx, V, dt):
    """ln p = -infinity: e^r - r - 1 is +infinity, and so are the loss with a KL term and the
    statistic; without one the loss is the others'."""
    b, lp = rows(V, dt, V + 2)
    z = b.z.copy()
    z[1, b.tok[1]] = -np.inf
    b.set(z)
    lp = np.where(np.arange(4) == 1, -3.0, tl.logprob(b.z, b.tok)[0])
    old, adv, ref = lp + 0.1, [1, 1, -1, 2], lp + 0.2
    logp, stats = ppo(ctx, b, old, adv, ref_logp=ref, kl_coef=0.1)
    assert logp[1] == -np.inf and stats[1] == np.inf and stats[3] == np.inf and np.isfinite(stats[[0, 2, 4]]).all()
    _, alone = ppo(ctx, b, old, adv, ref_logp=ref)
    _, none = ppo(ctx, b, old, adv)
    assert np.isfinite(none).all() and np.array_equal(alone[[0, 1, 2, 4]], none[[0, 1, 2, 4]]) and alone[3] == np.inf


@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", LENGTHS)
def test_gradient_of_an_infinite_slope(ctx, V, dt, pad):
    """Where the slope at ln p exceeds fp32, or is infinite (a masked token with a KL term), the
    entries go to the infinity of their sign, masked ones stay 0, and other rows are as ever."""
    b, lp = rows(V, dt, V + 3, pad)
    z = b.z.copy()
    z[2, b.tok[2]] = -np.inf
    b.set(z)
    lp, p, _, _ = tl.rows(b.z)
    lp = lp[np.arange(4), b.tok]
    old, ref = np.where(np.isfinite(lp), lp, -3) + 0.1, np.where(np.isfinite(lp), lp, -3) + [0, 200, 0, 0]
    masked = np.isneginf(b.z)
    one = np.zeros_like(b.z, bool)
    one[np.arange(4), b.tok] = True
    (_, plain), (_, g) = b.grad(), b.grad(pad=2 * pad)
    ppo(ctx, b, old, [1, 1, 1, -1], plain, ref_logp=np.where(np.arange(4) % 3 == 0, ref, 0), kl_coef=0.1)
    keep = b.logits.clone()
    for out in (g, b.logits):
        ppo(ctx, b, old, [1, 1, 1, -1], out, ref_logp=ref, kl_coef=0.1)
        got = out.double().cpu().numpy()
        b.logits.copy_(keep)
        assert bool((out[[0, 3]] == plain[[0, 3]]).all()) if out is g else True
        for i in (1, 2):
            assert np.isneginf(got[i, one[i]]).all()
            assert (got[i, masked[i] & ~one[i]] == 0).all()
            assert np.isposinf(got[i, ~masked[i] & ~one[i]]).all()
    # a ratio past fp32 with a negative advantage: the slope is -rho A = +infinity
    ppo(ctx, b, old - [0, 200, 0, 0], [0, -1, 0, 0], g, entropy_coef=0.1)
    got = g.double().cpu().numpy()
    assert np.isposinf(got[1, one[1]]).all() and np.isneginf(got[1, ~masked[1] & ~one[1]]).all()
    assert (got[masked & ~one] == 0).all()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("V", LENGTHS)
def test_pair_with_a_masked_rejected_token(ctx, V, dt):
    """D = +infinity: the loss is 0 without label smoothing, +infinity with it."""
    b, lp = rows(V, dt, V + 4)
    z = b.z.copy()
    z[1, b.tok[1]] = -np.inf
    b.set(z)
    off = np.array([0, 1, 2, 3, 4], np.int64)
    ref = np.where(np.isfinite(lp), lp, -3) - [0.3, 0, 0.5, -0.2]
    _, g = b.grad()
    reward, stats = empty(4), empty(5)

    def call(smooth):
        ctx.learn_token_pref(b.logits, cuda(b.tok), cuda(off), g, stats, ref_logp=cuda(ref.astype(np.float32)),
                             reward_out=reward, beta=0.5, label_smoothing=smooth, grad_scale=1024.0)
        ctx.sync()
        return stats.cpu().numpy(), reward.cpu().numpy(), g.double().cpu().numpy()
    s, r, got = call(0.0)
    wL, wg, wr, _, ws = tl.pref(b.z, b.tok, off, ref.astype(np.float32).astype(np.float64), 0.5, 0.0)
    assert np.isfinite(wL) and wr[1] == r[1] == -np.inf and s[4] == -np.inf
    np.testing.assert_allclose(s[:4], ws[:4], rtol=0, atol=1e-4)                    # ln p to 5e-5 at 150,001 entries
    np.testing.assert_allclose(r[[0, 2, 3]], wr[[0, 2, 3]], rtol=0, atol=1e-4)
    assert not got[:2].any()
    wg = wg * 1024
    one = np.arange(V) == b.tok[:, None]
    tol = 1e-4 * (np.abs(wg) + np.abs(wg).max() * one)
    assert (np.abs(got - wg) <= tol + HALF_ULP[dt] * (np.abs(wg) + tol) + TINY[dt]).all()
    s, r, _ = call(0.25)
    assert s[1] == np.inf and r[1] == -np.inf
