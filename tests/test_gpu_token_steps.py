"""The operators of a token policy's step as they are used: a rollout and a training step with all of
them in a row, captured and replayed calls, two contexts at once, and the ends of the draw's inputs."""
import threading

import numpy as np
import pytest

from gpu_util import context, need_gpu
from oracle import token_loss as tl
from oracle import token_rollout as tr
from test_gpu_token_losses import DTYPES, U, Batch, close, cuda, empty, grad_close, ttype
from test_gpu_token_rollout import Draw, check_top, host, ints, list_tol
from test_gpu_token_scores import Scores

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


# ---------------------------------------------------------------- a rollout and a training step

class Step:
    """logits = dropout(x) W for answers of `length` tokens; a loss of the tokens' ln p, the entropies and
    the listed entries' ln p. sequence and step name a row wherever it stands."""
    n, d, V, length, top, p, seed, site = 12, 40, 300, 5, 6, 0.25, 0xABCDEF0123456789, 4

    def __init__(self):
        rng = np.random.default_rng(7)
        rows = self.n * self.length
        self.x = rng.normal(size=(rows, self.d)).astype(np.float32)
        self.W = (rng.normal(size=(self.d, self.V)) * 0.4).astype(np.float32)
        self.seq = np.repeat(rng.integers(0, 2 ** 45, self.n), self.length)
        self.at = np.tile(np.arange(self.length, dtype=np.int32), self.n)
        self.rng = rng

    def hidden(self, ctx, rows):
        import torch
        x = cuda(self.x[rows])
        h = torch.empty_like(x)
        ctx.dropout(x, h, self.p, self.seed, self.site, cuda(self.seq[rows]), cuda(self.at[rows]))
        return h


def test_rollout_and_training_step(ctx):
    """The rollout takes a position of all answers at a time, the learner the whole batch in another
    order. Each operator's result against the 64-bit oracle on what it was given, and the
    gradients of W and x against those of the whole chain in 64 bits.

    With ez the error of a logit's sum of d products (d + 3 roundings of their sizes), p moves by
    a factor of 2 ez, ln p by 2 ez, H by 4 H ez; a product's sums of m terms add (m + 3) u of their sizes."""
    import torch
    s = Step()
    n, L, V, d = s.n, s.length, s.V, s.d
    W = cuda(s.W)
    ended = s.rng.integers(2, L + 1, n)
    tokens, old = np.full((n, L), -1, np.int32), np.zeros((n, L), np.float32)
    agent = dict(seed=s.seed, agent=3, top_k=50, top_p=0.9, temperature=0.8)
    for t in range(L):
        rows = np.arange(n) * L + t
        z = s.hidden(ctx, rows) @ W
        token = cuda(np.where(t < ended, 0, -1).astype(np.int32))
        lp, drawn = empty(n), empty(n)
        ctx.token_sample(z, token, lp, draw_logp_out=drawn, tokens=token, sequence=cuda(s.seq[rows]), step=cuda(s.at[rows]), **agent)
        ctx.sync()
        tokens[:, t], old[:, t] = host(token), host(lp)
        assert ((host(token) >= 0) == (t < ended)).all() and (host(drawn) >= host(lp)).all()
    # ---- the learner: rows in another order
    order = s.rng.permutation(n * L)
    tok, T = tokens.reshape(-1)[order], agent["temperature"]
    h = s.hidden(ctx, order)
    z = h @ W
    b = Batch(n * L, V, "f32", 1, T=T, out=0.0)
    b.set(z.double().cpu().numpy())
    b.tok, b.live_tok = tok, np.maximum(tok, 0)
    live = tok >= 0
    ids, top_lp, logp, H = ints(n * L, s.top), empty(n * L, s.top), empty(n * L), empty(n * L)
    ctx.token_top(b.logits, ids, top_lp, cuda(tok), logp, H, temperature=T)
    ctx.sync()
    want_ids, want_lp = tr.top(b.z, s.top, T, ~live)
    np.testing.assert_array_equal(host(ids), want_ids)
    x64, W64 = s.x[order].astype(np.float64), s.W.astype(np.float64)
    keep = tr.dropout_keep(d, s.p, s.seed, s.site, s.seq[order], s.at[order])
    h64 = np.where(keep, x64 * 65536 / (65536 - tr.dropout_least(s.p)), 0)
    close(h, h64, 2 * U * np.abs(h64) * (1 + U), "hidden")
    size = np.abs(h64) @ np.abs(W64)
    ez = ((d + 3) * U * size).max(axis=1, keepdims=True) / b.T
    # unchanged weights: the learner's ln p are the rollout's, each within both sides' errors
    t = b.tols()
    assert (np.abs(host(logp) - old.reshape(-1)[order])[live] <= (2 * (2 * ez[:, 0] + t["logp"]))[live]).all()
    # ---- the gradient: slopes at ln p, H and the list, then back through W and the dropout
    sc = Scores(b)
    sc.ids, sc.h = host(ids), s.rng.normal(size=(n * L, s.top)).astype(np.float32)
    dz = torch.empty_like(z)
    sc.call(ctx, b, dz)
    want, gt = sc.want(b)
    grad_close(b, dz, want, gt)
    dW, dh = h.t() @ dz, dz @ W.t()
    dx = torch.empty_like(dh)
    ctx.dropout(dh, dx, s.p, s.seed, s.site, cuda(s.seq[order]), cuda(s.at[order]))
    ctx.sync()
    z64 = h64 @ W64
    dz64 = tr.scores(z64, tok, sc.g, sc.e, sc.ids, sc.h, b.T)
    lp, p, ent, _ = tl.rows(z64, b.T)
    total = (np.abs(sc.g) * live)[:, None] + np.where(sc.ids >= 0, np.abs(sc.h), 0).sum(1, keepdims=True)
    e, ent = np.abs(sc.e)[:, None], ent[:, None]
    edz = gt + 2 * U * np.abs(want) + 1.01 * ez / b.T * p * (2 * total + e * (2 * (np.abs(lp) + ent) + 2 + 4 * ent))
    edz = np.where(live[:, None], edz, 0)
    ah, aW, adz = np.abs(h64), np.abs(W64), np.abs(dz64)
    close(dW, h64.T @ dz64, 1.01 * (ah.T @ edz + (n * L + 6) * U * (ah.T @ adz)), "dW")
    scale = keep * 65536 / (65536 - tr.dropout_least(s.p))
    close(dx, scale * (dz64 @ W64.T), 1.01 * scale * (edz @ aW.T + (V + 6) * U * (adz @ aW.T)), "dx")


# ---------------------------------------------------------------- graphs, threads

# a thread a row, a warp a row, blocks, clusters, streams of many rows
SIZES = [(500, 15, "f32"), (9, 300, "bf16"), (5, 40_000, "bf16"), (700, 9001, "f16"), (3, 151_111, "f32")]


def step_calls(c, n, V, dt, K, seed=0):
    """(calls, outputs) of every operator on one batch."""
    import torch
    b = Batch(n, V, dt, n + V + seed, pad=2)
    tok, u = cuda(b.tok), cuda(b.rng.random(n).astype(np.float32))
    seq, step = torch.arange(n, device="cuda") + 2 ** 33, torch.full((n,), 5, dtype=torch.int32, device="cuda")
    slope, listed = cuda(b.rng.normal(size=n).astype(np.float32)), cuda(b.rng.normal(size=(n, K)).astype(np.float32))
    ids, lp, logp, H, rank = ints(n, K), empty(n, K), empty(n), empty(n), ints(n)
    tokens, dl = [ints(n) for _ in range(3)], [empty(n) for _ in range(3)]
    grads, drop = [b.grad()[1] for _ in range(2)], torch.empty_like(b.logits)
    calls = [lambda: c.token_top(b.logits, ids, lp, tok, logp, H, rank),
             lambda: c.token_sample(b.logits, tokens[0], draw_logp_out=dl[0], tokens=tok, uniform=u),
             lambda: c.token_sample(b.logits, tokens[1], draw_logp_out=dl[1], tokens=tok, uniform=u, top_k=K, top_p=0.9),
             lambda: c.token_sample(b.logits, tokens[2], draw_logp_out=dl[2], sequence=seq, step=step, seed=5, top_k=K),
             lambda: c.learn_token_scores(b.logits, tok, grads[0], slope, slope),
             lambda: c.learn_token_scores(b.logits, tok, grads[1], slope, ids=ids, top_grad=listed),
             lambda: c.dropout(b.logits, drop, 0.1, 9, sequence=seq, step=step, residual=grads[0])]
    return calls, [ids, lp, logp, H, rank, *tokens, *dl, *grads, drop]


def test_captured_steps_replay_among_other_calls():
    """A graph of every operator, replayed between larger calls of the same context, and with inputs
    that changed in place."""
    torch = need_gpu()
    from paper_2106_07551_gb300 import Context
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), Context(0, stream) as c:
        calls, outs = [], []
        for size in SIZES:
            more, o = step_calls(c, *size, K=9)
            calls += more
            outs += o
        run = lambda: [f() for f in calls]  # noqa: E731
        run()
        c.sync()
        want = [x.clone() for x in outs]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        larger, _ = step_calls(c, 3000, 20_000, "bf16", 200)
        for _ in range(2):
            for x in outs:
                x.fill_(7)
            for f in larger:
                f()
            graph.replay()
            for f in larger:
                f()
            c.sync()
            assert all(bool((x == w).all()) for x, w in zip(outs, want))


def test_two_contexts_at_once():
    """Two threads with streams of their own, whose calls need different amounts of shared memory: each
    gives what it gives alone."""
    torch = need_gpu()
    from paper_2106_07551_gb300 import Context
    bad = []

    def work(sizes, K):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream), Context(0, stream) as c:
                batches = [step_calls(c, *size, K=K) for size in sizes]
                for calls, _ in batches:
                    for f in calls:
                        f()
                c.sync()
                want = [[x.clone() for x in outs] for _, outs in batches]
                start.wait()
                for _ in range(60):
                    for calls, _ in batches:
                        for f in calls:
                            f()
                c.sync()
                bad.extend("values" for (_, outs), w in zip(batches, want)
                           if not all(bool((x == y).all()) for x, y in zip(outs, w)))
        except Exception as e:                       # noqa: BLE001
            bad.append(repr(e))
            start.abort()

    start = threading.Barrier(2)
    threads = [threading.Thread(target=work, args=a) for a in (([(400, 30_000, "bf16"), (3, 151_111, "f32")], 600),
                                                               ([(350, 9001, "bf16"), (5, 120_000, "f32")], 200))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad


# ---------------------------------------------------------------- ends of the inputs

@pytest.mark.parametrize("n,V", [(40, 15), (9, 300), (5, 5003), (3, 151_111), (400, 9001)])
def test_random_numbers_past_the_ends(ctx, n, V):
    """1, more, and NaN draw the last entry that can be drawn; 0 the first."""
    b = Batch(n, V, "bf16", V, masked=0.3, out=0.0)
    lp, p, _, _ = tl.rows(b.z)
    for k in (0, 9):
        got = {}
        for u in (0.0, 1.0, 1.5, float("inf"), float("nan")):
            token = ints(n)
            ctx.token_sample(b.logits, token, uniform=cuda(np.full(n, u, np.float32)), top_k=k)
            ctx.sync()
            got[u] = host(token)
            assert (p[np.arange(n), got[u]] > 0).all()
        for u in (1.5, float("inf")):
            np.testing.assert_array_equal(got[u], got[1.0])
        nan = [v for u, v in got.items() if u != u][0]
        np.testing.assert_array_equal(nan, got[1.0])
        for i in range(n):
            order = tr.kept(b.z[i], k, 1.0)[0]
            order = order[p[i, order] > 0]
            assert got[0.0][i] == order[0] and got[1.0][i] == order[-1]


@pytest.mark.parametrize("n,V", [(1, 9000), (1, 200_000), (3, 60_001), (400, 9001), (600, 40_000)])
def test_entries_too_small_to_be_drawn(ctx, n, V):
    """Long runs of entries at 2^-127 of the largest, whose sums are not 0: one of the others is drawn, at
    both ends of the random numbers."""
    b = Batch(n, V, "f32", 1, out=0.0)
    z = np.full((n, V), -88.2)                           # times log2(e): -127.2
    z[:, V // 2 + 5] = 0.0
    z[:, V // 2 + 9] = -1.0
    z[: n // 2, -1] = -86.0
    b.set(z)
    for u, at in ((0.0, V // 2 + 5), (0.5, V // 2 + 5), (0.99, V // 2 + 9), (1.0, None)):
        token, dl = ints(n), empty(n)
        ctx.token_sample(b.logits, token, draw_logp_out=dl, uniform=cuda(np.full(n, u, np.float32)))
        ctx.sync()
        got = host(token)
        assert np.isin(got, [at] if at else [V // 2 + 9, V - 1]).all(), (u, got)
        assert np.isfinite(host(dl)).all()


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("V", [13, 700, 9001, 60_000])
def test_masks_of_the_lowest_value(ctx, V, dt):
    """Entries masked by the type's lowest value are listed last and never drawn, whatever the others
    are; a row of nothing else is uniform."""
    import torch
    low = float(torch.finfo(ttype(dt)).min)
    b = Batch(6, V, dt, V, out=0.0)
    z = b.z.copy()
    z[:, ::2] = low
    z[1], z[2, :], z[2, V // 2] = low, low, -1e4
    b.set(z)
    b.tok[:] = b.live_tok = np.array([1, 5, V // 2, 3, 7, 1], np.int32)
    check_top(ctx, b, min(V, 20))
    for k in (0, 20):
        for u in (None, np.zeros(6), np.full(6, np.float32(1 - 2.0 ** -24))):
            Draw(ctx, b, k, 1.0, u).check()
