"""Lists and draws of the longest rows, in batches whose rows are a CTA's each: sums that keep their
roundings' errors, maxima of many vectors, as many segments as a row can have. One row is given n
times (stride 0), so that it takes little memory and the oracle sorts it once."""
import numpy as np
import pytest

from gpu_util import context
from oracle import token_loss as tl
from oracle import token_rollout as tr
from test_gpu_token_draw_batches import check_running
from test_gpu_token_list_ways import rows_of
from test_gpu_token_losses import U, Batch, close, cuda, empty
from test_gpu_token_rollout import host, ints, list_tol

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


# a CTA a row with fine maxima, with larger groups, with few and many places; clusters; the longest rows
LISTS = [(400, 151_111, "f32", 64), (1300, 151_111, "f32", 700), (400, 300_001, "bf16", 64), (400, 600_001, "f32", 64),
         (1300, 1_200_007, "bf16", 300), (400, 600_001, "f16", 1024), (260, 4_000_003, "bf16", 100), (3, 2 ** 24, "f32", 50),
         (250, 2 ** 24, "bf16", 1)]


@pytest.mark.parametrize("kind", ["plain", "rising", "rounded", "few"])
@pytest.mark.parametrize("n,V,dt,K", LISTS)
def test_lists_of_long_rows(ctx, n, V, dt, K, kind):
    b = Batch(1, V, dt, V + K, out=0.0, shift=V % 3)
    rows_of(kind, b, K)
    z = b.logits.expand(n, V)
    token = int(np.flatnonzero(b.z[0] > -np.inf)[-1])
    ids, lp, rank, logp, H = ints(n, K), empty(n, K), ints(n), empty(n), empty(n)
    ctx.token_top(z, ids, lp, cuda(np.full(n, token, np.int32)), logp, H, rank)
    ctx.sync()
    want, wl = tr.top(b.z, K)
    got = host(ids)
    assert (got == want).all(), np.argwhere(got != want)[:5]
    assert (host(rank) == tr.rank(b.z, np.array([token]))).all()
    b.tok[:] = b.live_tok = np.array([token], np.int32)
    tol, t = list_tol(b)[0], b.tols()
    have = want[0] >= 0
    d = np.abs(host(lp).astype(np.float64)[:, have] - wl[0, have])
    assert (d <= tol[want[0, have]]).all() and np.isneginf(host(lp)[:, ~have]).all()
    close(logp, tl.rows(b.z)[0][0, token], t["logp"][0], "logp")
    close(H, tl.rows(b.z)[2][0], t["eH"][0], "entropy")


# the stream with its sums' errors, clusters, blocks of rows past the stream's longest, the longest rows
DRAWS = [(400, 70_001, "f32"), (400, 151_111, "f32"), (400, 300_001, "bf16"), (700, 131_073, "f16"), (3, 2 ** 24, "f32"),
         (300, 4_200_001, "f32"), (260, 8_400_003, "bf16"), (250, 2 ** 24, "f32"), (40, 1_000_003, "bf16")]


@pytest.mark.parametrize("masked", [0.0, 0.9])
@pytest.mark.parametrize("n,V,dt", DRAWS)
def test_draws_of_long_rows(ctx, n, V, dt, masked):
    b = Batch(1, V, dt, V + n, T=1.1, masked=masked, out=0.0, shift=V % 3)
    u = b.rng.random(n).astype(np.float32)
    u[0] = 0.0
    token, lp, H, dl = ints(n), empty(n), empty(n), empty(n)
    ctx.token_sample(b.logits.expand(n, V), token, lp, H, dl, uniform=cuda(u), temperature=b.T)
    ctx.sync()
    got = host(token)
    check_running(b, u.astype(np.float64), got)
    b.tok[:] = b.live_tok = got[:1]
    tol = list_tol(b)[0][got]
    want = tl.rows(b.z, b.T)[0][0, got]
    assert (np.abs(host(lp) - want) <= tol).all() and (host(dl) == host(lp)).all()
    close(H, tl.rows(b.z, b.T)[2][0], b.tols()["eH"][0], "entropy")
