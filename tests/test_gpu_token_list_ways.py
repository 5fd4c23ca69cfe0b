"""Lists and draws at the sizes that decide how a row is listed: a warp, a block or a cluster a row, groups
or entries that give the bound, slices that list a share each. One row is given n times (stride 0),
so that the oracle sorts it once. Ids are equal; ln p is within the rollout tests' bounds."""
import numpy as np
import pytest

from gpu_util import context
from oracle import token_rollout as tr
from test_gpu_token_losses import DTYPES, Batch, cuda, empty
from test_gpu_token_rollout import host, ints, list_tol

pytestmark = pytest.mark.gpu

WAYS = [(164, 184_696, "f32", 1), (333, 151_111, "f32", 64), (333, 151_111, "f32", 700), (54, 151_120, "bf16", 56),
        (1, 131_072, "bf16", 20), (1, 131_072, "f16", 100), (3, 262_144, "bf16", 1024), (200, 250_000, "bf16", 10),
        (92, 8163, "bf16", 844), (1, 5510, "f16", 439), (300, 20_000, "bf16", 200), (20, 66_000, "f32", 1000),
        (700, 40_001, "f32", 300), (2000, 12_000, "f16", 128), (40, 2041, "bf16", 1024), (40, 1021, "f32", 1000),
        (40, 500, "f16", 129), (40, 300, "f32", 250), (40, 500, "bf16", 128), (40, 255, "f32", 65), (40, 100, "f32", 33),
        (40, 2041, "f16", 65), (900, 65_536, "bf16", 64), (400, 70_001, "f16", 500)]


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


def rows_of(kind, b, K):
    z = b.z.copy()
    if kind == "rising":                             # the first entries in the last slice, and beside one another
        z[0] = np.sort(z[0])
    elif kind == "rounded":                          # many equal ones
        z[0] = np.round(z[0])
    elif kind == "equal":
        z[0] = -1.5
    elif kind == "few":                              # fewer than the list has places
        z[0, b.rng.permutation(b.V)[K // 2 + 1:]] = -np.inf
    b.set(z)


@pytest.mark.parametrize("kind", ["plain", "rising", "rounded", "equal", "few"])
@pytest.mark.parametrize("n,V,dt,K", WAYS)
def test_ways(ctx, n, V, dt, K, kind):
    b = Batch(1, V, dt, V + K, out=0.0, pad=0, shift=1 if V % 2 else 0)
    rows_of(kind, b, K)
    z = b.logits.expand(n, V)
    token = int(np.flatnonzero(b.z[0] > -np.inf)[-1])
    tok = np.full(n, token, np.int32)
    ids, lp, rank = ints(n, K), empty(n, K), ints(n)
    ctx.token_top(z, ids, lp, cuda(tok), rank_out=rank)
    u = np.linspace(0, 1, n, endpoint=False).astype(np.float32)
    drawn, dl = ints(n), empty(n)
    ctx.token_sample(z, drawn, draw_logp_out=dl, uniform=cuda(u), top_k=K)
    ctx.sync()
    want, wl = tr.top(b.z, K)
    got = host(ids)
    assert (got == want).all(), np.argwhere(got != want)[:5]
    assert (host(rank) == tr.rank(b.z, tok[:1])).all()
    b.tok[:] = b.live_tok = np.array([token], np.int32)
    tol = list_tol(b)[0]
    have = want[0] >= 0
    d = np.abs(host(lp).astype(np.float64)[:, have] - wl[0, have])
    assert (d <= tol[want[0, have]]).all() and np.isneginf(host(lp)[:, ~have]).all()
    # the draws: their places in the list do not fall as the random numbers rise
    place = np.full(V, -1)
    place[want[0, have]] = np.arange(have.sum())
    at = place[host(drawn)]
    assert (at >= 0).all() and (np.diff(at) >= 0).all() and at[0] == 0
    assert np.isfinite(host(dl)).all()
