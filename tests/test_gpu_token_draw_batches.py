"""A row's draw does not depend on the batch that it is in: the same logits and random numbers give the same
token alone, among a few rows (which are shared by several CTAs) or thousands (which pass as a
stream), and wherever the row lies in memory. Tokens are equal; their interval of the running
probability holds the random number within what fp32 sums may lose."""
import numpy as np
import pytest

from gpu_util import context
from oracle import token_loss as tl
from oracle import token_rollout as tr
from test_gpu_token_losses import DTYPES, U, Batch, cuda, empty
from test_gpu_token_rollout import host, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


def draws(ctx, z, u, n, T, **more):
    """Tokens by calls of n rows each."""
    token, rows = ints(len(u)), z.expand(n, z.shape[1])
    for i in range(0, len(u), n):
        m = min(n, len(u) - i)
        ctx.token_sample(rows[:m], token[i:i + m], uniform=u[i:i + m], temperature=T, **more)
    return token


def check_running(b, u, token, exact=None):
    """The 64-bit running probability at the tokens, within four times p's error and the sums'."""
    _, p, _, _ = tl.rows(b.z, b.T)
    p = p[0]
    eps = 4 * float((b.tols()["ep"][0] * p).sum()) + 40 * U
    cum = np.cumsum(p)
    assert (token >= 0).all() and (p[token] > 0).all()
    assert (cum[token] - p[token] - eps <= u).all() and (u <= cum[token] + eps).all()


# lengths of a warp a row, of a block or cluster a row, of the stream; odd ones are not aligned alike in a batch
CASES = [(100, "f32", 20_000), (255, "bf16", 20_000), (1021, "f32", 20_000), (1999, "bf16", 20_000), (2041, "f16", 20_000),
         (5003, "bf16", 4000), (9001, "f32", 4000), (50_001, "f16", 3000), (131_072, "bf16", 3000), (70_001, "f32", 3000),
         (151_111, "f32", 3000), (300_001, "bf16", 2000)]


@pytest.mark.parametrize("V,dt,count", CASES)
def test_draws_of_any_batch(ctx, V, dt, count):
    import torch
    b = Batch(1, V, dt, V, T=0.9, masked=0.1 if V % 2 else 0.0, out=0.0)
    u = b.rng.random(count).astype(np.float32)
    u[:3] = [0.0, np.float32(1 - 2.0 ** -24), 1e-30]
    at = cuda(u)
    want = draws(ctx, b.logits, at, count, b.T)
    ctx.sync()
    check_running(b, np.minimum(u, 1.0).astype(np.float64), host(want))
    for n in (30, 75, 130, 240, 700):
        m = min(count, 100 * n)
        got = draws(ctx, b.logits, at[:m], n, b.T)
        ctx.sync()
        assert int((got != want[:m]).sum()) == 0, (n, int((got != want[:m]).sum()))
    # at other places in memory
    room = torch.zeros(V + 64, dtype=b.logits.dtype, device="cuda")
    for shift in (1, 2, 3, 5, 7):
        moved = room[shift:shift + V].view(1, V)
        moved.copy_(b.logits)
        for n in (count, 20):
            m = min(count, 100 * n)
            got = draws(ctx, moved, at[:m], n, b.T)
            ctx.sync()
            assert int((got != want[:m]).sum()) == 0, (shift, n, int((got != want[:m]).sum()))


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("V", [13, 333, 1501, 5003, 20_001, 90_001])
def test_rows_of_a_batch_alone(ctx, V, dt):
    """Rows one after another without a gap, each again in a call of its own, by the numbers of their
    sequences and steps; from all entries and from the first of a list."""
    n = 40 if V > 50_000 else 200
    b = Batch(n, V, dt, V, out=0.0)
    seq = b.rng.integers(0, 2 ** 40, n)
    step = b.rng.integers(0, 100, n).astype(np.int32)
    for k, p in ((0, 1.0), (min(V, 40), 0.9)):
        args = dict(seed=77, agent=3, top_k=k, top_p=p)
        whole, alone = ints(n), ints(n)
        ctx.token_sample(b.logits, whole, sequence=cuda(seq), step=cuda(step), **args)
        s, t = cuda(seq), cuda(step)
        for i in range(0, n, 3):
            ctx.token_sample(b.logits[i:i + 1].clone(), alone[i:i + 1], sequence=s[i:i + 1], step=t[i:i + 1], **args)
        ctx.sync()
        np.testing.assert_array_equal(host(whole)[::3], host(alone)[::3])
        u = tr.token_uniform(77, seq, step, 3)
        by_u = ints(n)
        ctx.token_sample(b.logits, by_u, uniform=cuda(u.astype(np.float32)), top_k=k, top_p=p)
        ctx.sync()
        np.testing.assert_array_equal(host(by_u), host(whole))
