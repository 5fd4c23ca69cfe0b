"""Gradients of scores at slopes that are not finite, by every kernel that takes rows of a length, without
a list, and with lists that have the token among their entries or not. No tolerances: an entry is
NaN or the infinity of its sign."""
import numpy as np
import pytest

from gpu_util import context
from test_gpu_token_losses import Batch, cuda

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
ROWS = 12


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


def call(ctx, b, g, e=None, ids=None, h=None):
    opt = lambda x, t: None if x is None else cuda(np.asarray(x, t))  # noqa: E731
    _, out = b.grad()
    ctx.learn_token_scores(b.logits, cuda(b.tok), out, opt(g, np.float32), opt(e, np.float32), opt(ids, np.int32),
                           opt(h, np.float32))
    ctx.sync()
    return out.double().cpu().numpy()


def batch(V, dt="f32", n=ROWS):
    b = Batch(n, V, dt, V, masked=0.3, out=0.0)
    z = b.z.copy()
    at = np.arange(n)
    for i in range(1, 4):                                # the entries that are listed are not masked
        z[at, (b.tok + i) % V] = 1.0
    b.set(z)
    return b


# a thread a row, registers, shared memory, the ring with one CTA a row, clusters
LENGTHS = [20, 300, 2500, 9000, 70_000, 300_000]


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("V", LENGTHS)
def test_slopes_at_the_entropy(ctx, V, listed):
    """An infinite or NaN slope at H makes the whole row NaN, whatever the others are."""
    b = batch(V)
    g = np.linspace(-1, 1, ROWS)
    e = np.array([INF, -INF, NAN, 0.5, INF, -INF, NAN, 0.0, INF, NAN, -INF, 1.0])
    g[4:8] = [INF, INF, -INF, INF]
    g[8:11] = NAN
    ids = h = None
    if listed:
        ids, h = (b.tok[:, None] + np.arange(1, 4)) % V, np.ones((ROWS, 3))
        h[4], h[5, 1] = [INF, 2.0, -1.0], -INF
    got = call(ctx, b, g, e, ids, h)
    for i in (0, 1, 2, 4, 5, 6, 8, 9, 10):
        assert np.isnan(got[i]).all(), (i, got[i][~np.isnan(got[i])][:5])
    for i in (3, 11):
        assert np.isfinite(got[i]).all()
    only = call(ctx, b, None, e)
    assert np.isnan(only[[0, 1, 2, 4, 5, 6, 8, 9, 10]]).all() and np.isfinite(only[[3, 7, 11]]).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", LENGTHS)
def test_infinities_of_both_signs(ctx, V, dt):
    """Infinite slopes of both signs among the token and the list, or a NaN, make the whole row NaN; of one
    sign they have the infinity of their sign where they stand, and the other entries the other."""
    b = batch(V, dt)
    ids = (b.tok[:, None] + np.arange(1, 4)) % V
    g, h = np.ones(ROWS), np.ones((ROWS, 3))
    g[0], h[0, 1] = INF, -INF
    g[1], h[1, 2] = -INF, INF
    h[2] = [INF, -INF, 0]
    h[3, 0] = NAN
    g[4] = NAN
    ids[5, :2], h[5, :2] = b.tok[5], [-INF, 1]               # the token's own two
    g[5] = INF
    ids[6, 1], h[6, :2] = ids[6, 0], [INF, -INF]             # one id's two
    g[7], h[7, 0] = INF, NAN
    g[8], h[8, 0] = INF, INF
    ids[9, 2], g[9], h[9, 2] = b.tok[9], -INF, -INF
    h[10, 1], ids[10, 1] = NAN, -1                           # an absent entry has no slope
    got = call(ctx, b, g, None, ids, h)
    for i in range(8):
        assert np.isnan(got[i]).all(), (i, got[i][~np.isnan(got[i])][:5])
    for i, at, sign in ((8, [b.tok[8], ids[8, 0]], 1), (9, [b.tok[9]], -1)):
        p = np.exp(b.z[i] - b.z[i].max())
        want = np.where(p > 0, -sign * INF, 0)
        want[at] = sign * INF
        np.testing.assert_array_equal(got[i], want)
    assert np.isfinite(got[10:]).all()


@pytest.mark.parametrize("top", [1, 31, 33, 200, 1024])
@pytest.mark.parametrize("V", [20, 300, 2500, 9000, 70_000, 300_000])
def test_slopes_of_one_id_are_added_in_their_order(ctx, V, top):
    """At a masked entry the gradient is the sum of its slopes: of all that are listed, in the list's order, then the
    token's. Equal to the bit: fp32 sums one after another."""
    n = 6
    b = Batch(n, V, "f32", V + top, out=0.0)
    z = b.z.copy()
    few = np.stack([b.rng.permutation(V)[:8] for _ in range(n)])
    z[np.arange(n)[:, None], few] = -np.inf              # eight masked entries, the token one of them
    z[np.arange(n), [next(j for j in range(V) if j not in set(f)) for f in few]] = 1.0
    b.tok[:] = few[:, 3]
    b.set(z)
    ids = few[np.arange(n)[:, None], b.rng.integers(0, 8, (n, top))]
    ids[0] = few[0, 3]                                   # the token alone
    ids[1, 1:] = -1                                      # once, and nothing else
    ids[2, ::2] = -1
    g, h = b.rng.normal(size=n).astype(np.float32), b.rng.normal(size=(n, top)).astype(np.float32)
    got = call(ctx, b, g, None, ids, h)
    for i in range(n):
        want = {}
        for j, x in list(zip(ids[i], h[i])) + [(b.tok[i], g[i])]:
            if j >= 0:
                want[j] = np.float32(want[j] + x) if j in want else x
        for j in few[i]:
            assert got[i, j] == want.get(j, 0.0), (i, j)
