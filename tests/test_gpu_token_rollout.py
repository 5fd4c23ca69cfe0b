"""Lists of the most likely entries and the draw of tokens against the 64-bit oracle. Ids, tokens
and ranks are equal; a drawn token's interval of the running probability holds the random number
within what the sums' roundings allow. The bounds of ln p and H are those of the losses' tests:
the row's sums are formed alike."""
import numpy as np
import pytest

from gpu_util import context, need_gpu
from oracle import token_loss as tl
from oracle import token_rollout as tr
from test_gpu_token_losses import DTYPES, U, Batch, close, cuda, empty, f32, ttype

pytestmark = pytest.mark.gpu

from paper_2106_07551_gb300 import MalibError


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


def ints(*shape):
    import torch
    return torch.full(shape, 99, dtype=torch.int32, device="cuda")


def host(x):
    return x.cpu().numpy()


def list_tol(b):
    """[n][V]: of ln p of every entry."""
    lp, p, _, _ = tl.rows(b.z, b.T)
    d = lp.max(axis=1, keepdims=True) - lp
    X = np.where(p > 0, p * np.where(p > 0, d, 0), 0).sum(axis=1, keepdims=True) / np.log(2)
    eS = 2.0 ** -22 + 2.1 * U * X + U * (b.V / 256 + 64)
    return eS + 4 * U * (1 + d - lp.max(axis=1, keepdims=True))


def run_top(ctx, b, K, tokens=True):
    ids, lp = ints(b.n, K), empty(b.n, K)
    logp, H, rank = empty(b.n), empty(b.n), ints(b.n)
    if tokens:
        ctx.token_top(b.logits, ids, lp, cuda(b.tok), logp, H, rank, temperature=b.T)
    else:
        ctx.token_top(b.logits, ids, lp, entropy_out=H, temperature=b.T)
    ctx.sync()
    return ids, lp, logp, H, rank


def check_top(ctx, b, K):
    ids, lp, logp, H, rank = run_top(ctx, b, K)
    left = b.tok < 0
    want_ids, want_lp = tr.top(b.z, K, b.T, left)
    np.testing.assert_array_equal(host(ids), want_ids)
    np.testing.assert_array_equal(host(rank), tr.rank(b.z, b.tok))
    bad = tr.broken(b.z)
    t = b.tols() if not bad.any() else None
    got = host(lp).astype(np.float64)
    np.testing.assert_array_equal(np.isneginf(got), np.isneginf(want_lp))
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want_lp))
    if t is None:
        np.testing.assert_array_equal(np.isnan(host(logp)), bad & ~left)
        return
    tol = list_tol(b)
    fin = np.isfinite(want_lp) & (want_ids >= 0)
    r, c = np.nonzero(fin)
    assert (np.abs(got[r, c] - want_lp[r, c]) <= tol[r, want_ids[r, c]]).all()
    assert (got[left] == 0).all()
    want, wH, live = tl.logprob(b.z, b.tok, b.T)
    with np.errstate(invalid="ignore"):
        same = (host(logp).astype(np.float64) == want) | (np.abs(host(logp) - want) <= np.where(live, t["logp"], 0))
    assert same.all()
    close(H, wH, np.where(live, t["eH"], 0), "entropy")


# rows of a few entries to long ones; 8,192 and 2,048 entries to either side of a warp's and a CTA's rows
SHAPES = [(3, 1), (7, 2), (64, 5), (33, 15), (9, 257), (5, 1000), (6, 2047), (6, 2055), (3, 4097), (5, 32768), (3, 50001)]


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("n,V", SHAPES + [(2, 151111), (700, 9001), (1300, 300)])
def test_top(ctx, n, V, dt):
    b = Batch(n, V, dt, 10 * V + n, pad=3, shift=1)
    for K in {1, 7, min(64, V + 3), min(1024, V)}:
        check_top(ctx, b, K)


@pytest.mark.parametrize("dt", DTYPES)
def test_top_masks_and_temperature(ctx, dt):
    b = Batch(12, 5003, dt, 5, T=0.37, masked=0.9)
    z = b.z.copy()
    z[2] = -np.inf                                   # left out
    z[3] = -np.inf
    z[3, [17, 4000]] = [1.0, 2.0]                    # fewer entries than the list
    z[4, :4000] = -np.inf
    z[5, b.live_tok[5]] = -np.inf                    # a masked token
    b.set(z)
    for K in (1, 5, 50, 1024):
        check_top(ctx, b, K)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("V", [37, 1500, 9001, 70_000])
def test_top_of_equal_values(ctx, V, dt):
    """More equal entries than are sorted: the lower indices come first. And ascending rows."""
    b = Batch(8, V, dt, V, pad=1)
    z = b.z.copy()
    rng = np.random.default_rng(V)
    z[0] = 0.0
    z[1] = rng.choice([-0.0, 0.0], V)                # equal as well
    z[2] = rng.choice([1.0, 1.0, 1.0, 2.0], V)
    z[3] = np.round(z[3])
    z[4] = np.sort(z[4])
    z[5] = -np.sort(-z[5])
    z[6] = -7.0
    z[6, V // 3:] = -np.inf
    z[7] = np.where(np.arange(V) % 64 < 32, 3.0, z[7])
    b.set(z)
    for K in (1, 30, min(V, 1000)):
        check_top(ctx, b, K)


@pytest.mark.parametrize("dt", DTYPES)
def test_top_extreme_values(ctx, dt):
    import torch
    b = Batch(9, 3000, dt, 9)
    big = float(torch.finfo(ttype(dt)).max)
    tiny = float(torch.finfo(ttype(dt)).tiny)
    z = b.z.copy()
    z[0, 5], z[1, 2999], z[2, 0] = np.nan, np.inf, big
    z[3] = -big
    z[4, ::2] = -big
    z[5] = np.random.default_rng(1).choice([-tiny, -tiny / 2, 0.0, tiny / 2, tiny], 3000)
    z[6], z[6, 7] = -np.inf, np.nan
    b.set(z)
    with np.errstate(invalid="ignore", over="ignore"):
        ids, lp, logp, H, rank = run_top(ctx, b, 40)
        want, wl = tr.top(b.z, 40, b.T, b.tok < 0)
        np.testing.assert_array_equal(host(ids), want)
        np.testing.assert_array_equal(host(rank), tr.rank(b.z, b.tok))
        np.testing.assert_array_equal(np.isnan(host(lp)), np.isnan(wl))


def test_top_without_tokens_shared_row_and_errors(ctx):
    import torch
    b = Batch(5, 700, "bf16", 3)
    ids, lp, _, H, _ = run_top(ctx, b, 9, tokens=False)
    want, wl = tr.top(b.z, 9, b.T)
    np.testing.assert_array_equal(host(ids), want)
    one = b.logits[:1].expand(40, 700)               # a row that all share
    ids, lp = ints(40, 9), empty(40, 9)
    ctx.token_top(one, ids, lp)
    ctx.sync()
    np.testing.assert_array_equal(host(ids), np.repeat(want[:1], 40, 0))
    b.tok[2] = 700                                   # past the vocabulary: left out, reported
    ids, lp, rank = ints(5, 9), empty(5, 9), ints(5)
    ctx.token_top(b.logits, ids, lp, cuda(b.tok), rank_out=rank)
    with pytest.raises(MalibError, match="EINVAL"):
        ctx.sync()
    assert (host(ids)[2] == -1).all() and host(rank)[2] == 0 and (host(lp)[2] == 0).all()
    ctx.token_top(b.logits[:0], ids[:0], lp[:0])
    ctx.sync()


class Draw:
    def __init__(self, ctx, b, top_k=0, top_p=1.0, u=None, **more):
        self.b, self.k, self.p = b, top_k, f32(top_p)
        n = b.n
        self.u = b.rng.random(n).astype(np.float32) if u is None else np.asarray(u, np.float32)
        self.token, self.lp, self.H, self.dl = ints(n), empty(n), empty(n), empty(n)
        if not more:
            more = dict(uniform=cuda(self.u))
        ctx.token_sample(b.logits, self.token, self.lp, self.H, self.dl, tokens=cuda(b.tok), top_k=top_k, top_p=top_p,
                         temperature=b.T, **more)
        ctx.sync()

    def check(self):
        b, t = self.b, self.b.tols()
        tol_lp = list_tol(b)
        lp, p, H, live = tl.rows(b.z, b.T)
        live = live & (b.tok >= 0)
        token, dl = host(self.token), host(self.dl).astype(np.float64)
        close(self.H, np.where(live, H, 0), np.where(live, t["eH"], 0), "entropy")
        for i in range(b.n):
            if not live[i]:
                assert token[i] == -1 and host(self.lp)[i] == 0 and dl[i] == 0
                continue
            j = token[i]
            assert 0 <= j < b.V and p[i, j] > 0, (i, j)
            assert abs(host(self.lp)[i] - lp[i, j]) <= tol_lp[i, j]
            # a running sum's error: every term's, and the additions'; of the whole at most
            eps = 4 * float((t["ep"][i] * p[i]).sum()) + 40 * U
            ok = False
            for slack in (0.0, eps, -eps):               # on which side of top_p an entry lies may be rounding
                ids, w = tr.kept(b.z[i], self.k, self.p, b.T, slack)
                at = np.flatnonzero(ids == j)
                if not len(at):
                    continue
                cum = np.cumsum(w) / w.sum()
                lo = cum[at[0]] - w[at[0]] / w.sum()
                u = min(float(self.u[i]), 1.0)
                if lo - eps / w.sum() <= u <= cum[at[0]] + eps / w.sum():
                    want = lp[i, j] - np.log(w.sum())
                    ok |= abs(dl[i] - want) <= tol_lp[i, j] + eps / w.sum() + 8 * U * (1 + abs(want))
            assert ok, (i, j, self.u[i], dl[i])


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("n,V", SHAPES + [(2, 151111), (700, 9001), (3000, 15), (1300, 300)])
def test_sample(ctx, n, V, dt):
    b = Batch(n, V, dt, 10 * V + n, pad=3, shift=1, T=0.8)
    Draw(ctx, b).check()
    Draw(ctx, b, 50, 0.95).check()
    Draw(ctx, b, min(V, 7)).check()
    if n < 100:
        Draw(ctx, b, 1024, 0.9).check()


@pytest.mark.parametrize("dt", DTYPES)
def test_sample_masks_and_ends(ctx, dt):
    b = Batch(12, 5003, dt, 5, T=1.3, masked=0.9)
    z = b.z.copy()
    z[2] = -np.inf
    z[3] = -np.inf
    z[3, [17, 4000]] = [1.0, 2.0]
    z[4, :4000] = -np.inf
    z[5] = -np.inf
    z[5, 5002] = -3.0
    z[6] = 1.5                                       # equal entries
    b.set(z)
    for k, p in ((0, 1.0), (20, 0.5), (1024, 0.99), (1, 1.0)):
        for u in (None, np.zeros(12), np.full(12, np.float32(1 - 2.0 ** -24)), np.ones(12), np.full(12, 0.5)):
            d = Draw(ctx, b, k, p, u)
            d.check()
            if k == 1:
                live = host(d.token) >= 0
                assert (host(d.dl)[live] == 0).all()


@pytest.mark.parametrize("k", [0, 30])
def test_sample_broken_rows_and_in_place(ctx, k):
    b = Batch(6, 3001, "bf16", 2, out=0.0)
    z = b.z.copy()
    z[1, 2], z[3, 3000] = np.nan, np.inf
    b.set(z)
    u = cuda(b.rng.random(6).astype(np.float32))
    tokens = cuda(np.array([5, 5, -1, 5, 9_999_999, 0], np.int32))   # values are not looked at
    dl = empty(6)
    want = ints(6)
    ctx.token_sample(b.logits, want, draw_logp_out=dl, tokens=tokens, uniform=u, top_k=k)
    ctx.token_sample(b.logits, tokens, tokens=tokens, uniform=u, top_k=k)
    ctx.sync()
    got = host(tokens)
    np.testing.assert_array_equal(got, host(want))
    assert (got[[1, 2, 3]] == -1).all() and (got[[0, 4, 5]] >= 0).all()
    np.testing.assert_array_equal(np.isnan(host(dl)), [False, True, False, True, False, False])


def test_sample_by_sequence(ctx):
    """The draws of a sequence and step are those of the generator, in whatever batch they are."""
    b = Batch(40, 1234, "f32", 8, out=0.0)
    seq = b.rng.integers(-2 ** 40, 2 ** 40, 40)
    step = b.rng.integers(0, 1000, 40).astype(np.int32)
    u = tr.token_uniform(0x1234567890ABCDEF, seq, step, 77)
    for k, p in ((0, 1.0), (40, 0.9)):
        args = dict(sequence=cuda(seq), step=cuda(step), seed=0x1234567890ABCDEF, agent=77)
        Draw(ctx, b, k, p, u, **args).check()
        whole = ints(40)
        ctx.token_sample(b.logits, whole, top_k=k, top_p=p, **args)
        part = ints(7)
        ctx.token_sample(b.logits[20:27], part, top_k=k, top_p=p, sequence=cuda(seq[20:27]), step=cuda(step[20:27]),
                         seed=args["seed"], agent=77)
        ctx.sync()
        np.testing.assert_array_equal(host(whole)[20:27], host(part))


def test_sample_frequencies(ctx):
    """2^18 draws of one row: every entry's count within six standard deviations."""
    import torch
    n, V = 2 ** 18, 11
    b = Batch(1, V, "f32", 4, masked=0.3, out=0.0)
    tok, step = ints(n), torch.zeros(n, dtype=torch.int32, device="cuda")
    ctx.token_sample(b.logits.expand(n, V), tok, sequence=torch.arange(n, device="cuda"), step=step, seed=5)
    ctx.sync()
    p = tl.rows(b.z)[1][0]
    count = np.bincount(host(tok), minlength=V)
    assert (np.abs(count - n * p) <= 6 * np.sqrt(n * p * (1 - p)) + 1e-9).all()


def test_refusals(ctx):
    import torch
    b = Batch(4, 100, "f32", 1)
    tok = cuda(b.tok)
    top = lambda ids=ints(4, 5), lp=empty(4, 5), **k: ctx.token_top(b.logits, ids, lp, **k)  # noqa: E731
    draw = lambda out=ints(4), **k: ctx.token_sample(b.logits, out, **{"uniform": empty(4), **k})  # noqa: E731
    for f in (lambda: top(ints(4, 5).long()), lambda: top(ints(5, 5), empty(5, 5)), lambda: top(lp=empty(4, 6)),
              lambda: top(tokens=tok.long()), lambda: top(tokens=tok, rank_out=empty(4)), lambda: draw(ints(3)),
              lambda: draw(uniform=empty(5)), lambda: ctx.token_top(b.logits.double(), ints(4, 5), empty(4, 5))):
        with pytest.raises(ValueError):
            f()
    cpu = torch.empty((4, 5), dtype=torch.int32)
    for f in (lambda: top(ints(4, 0), empty(4, 0)), lambda: top(ints(4, 1025), empty(4, 1025)), lambda: top(cpu),
              lambda: top(rank_out=ints(4)), lambda: top(logp_out=empty(4)), lambda: top(temperature=0.0),
              lambda: draw(top_k=-1), lambda: draw(top_k=1025), lambda: draw(top_p=0.5), lambda: draw(top_k=5, top_p=0.0),
              lambda: draw(top_k=5, top_p=1.5), lambda: draw(top_k=5, top_p=float("nan")), lambda: draw(agent=2 ** 31),
              lambda: draw(uniform=None), lambda: draw(cpu[:, 0].contiguous()), lambda: draw(temperature=float("inf"))):
        with pytest.raises(MalibError, match="EINVAL"):
            f()
    ctx.sync()
