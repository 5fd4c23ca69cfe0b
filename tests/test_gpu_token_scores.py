"""The gradient of any loss of log-probabilities and entropies, and dropout, against the 64-bit
oracle. The scores' bounds are those of the losses' tests: p is good to ep, ln p to its own bound,
a sum of K slopes to (K / 32 + 8) u of its terms, products and the last addition to some u."""
import numpy as np
import pytest

from gpu_util import context, need_gpu
from oracle import token_rollout as tr
from test_gpu_token_losses import DTYPES, HALF_ULP, TINY, U, Batch, close, cuda, empty, f32, grad_close, ttype

pytestmark = pytest.mark.gpu

from paper_2106_07551_gb300 import MalibError


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


class Scores:
    def __init__(self, b, logp=True, ent=True, top=0, ragged=0.3, twice=False):
        rng, n = b.rng, b.n
        self.g = rng.normal(size=n).astype(np.float32) if logp else None
        self.e = rng.normal(size=n).astype(np.float32) if ent else None
        self.ids = self.h = None
        if top:
            ids = np.stack([rng.permutation(max(b.V, top))[:top] % b.V for _ in range(n)])
            if twice:
                ids[:, -1] = ids[:, 0]
                ids[:, top // 2] = np.maximum(b.tok, 0)
            ids[rng.random(ids.shape) < ragged] = -1
            if n > 2:
                ids[2] = -1
            z = b.z.copy()
            for i in range(n):
                at = ids[i][ids[i] >= 0]
                z[i, at] = np.where(rng.random(len(at)) < 0.1, -np.inf, rng.normal(size=len(at)) * 2)
            z[np.arange(n), b.live_tok] = 1.0
            b.set(z)
            self.ids, self.h = ids.astype(np.int32), rng.normal(size=ids.shape).astype(np.float32)

    def call(self, ctx, b, g, scale=1.0, z=None):
        opt = lambda x: None if x is None else cuda(x)  # noqa: E731
        ctx.learn_token_scores(b.logits if z is None else z, cuda(b.tok), g, opt(self.g), opt(self.e), opt(self.ids),
                               opt(self.h), temperature=b.T, grad_scale=scale)

    def want(self, b):
        want = tr.scores(b.z, b.tok, self.g, self.e, self.ids, self.h, b.T)
        t, n = b.tols(), b.n
        p, live = t["p"], (b.tok >= 0) & ~np.isneginf(b.z).all(1)
        size, times = np.zeros_like(p), np.zeros_like(p)
        if self.g is not None:
            size[np.arange(n), np.maximum(b.tok, 0)] += np.abs(self.g)
        if self.ids is not None:
            for i in range(n):
                have = self.ids[i] >= 0
                np.add.at(size[i], self.ids[i][have], np.abs(self.h[i][have]))
                np.add.at(times[i], self.ids[i][have], 1)
        K = 0 if self.ids is None else self.ids.shape[1]
        total = size.sum(1, keepdims=True)               # the slopes' sizes: a bound of their sum, too
        gt = p * total * (t["ep"] + (K / 32 + 16) * U) + U * (4 + times) * size
        if self.e is not None:
            lpH = np.where(p > 0, np.abs(t["lp"]) + t["H"][:, None], 0)
            gt = gt + np.abs(self.e)[:, None] * p * (lpH * (t["ep"] + 6 * U) + t["eH"][:, None] + t["logp"][:, None])
        return want, np.where(live[:, None], (gt + 1e-37) / b.T, 0)


def check_scores(ctx, b, pad=0, shift=0, **kw):
    s = Scores(b, **kw)
    scale = 4096.0 if b.dt == "f16" else 1.0
    buf, g = b.grad(pad, shift)
    s.call(ctx, b, g, scale)
    ctx.sync()
    grad_close(b, g, *s.want(b), scale)
    if pad:                                              # what lies between the rows stays
        assert bool((buf[shift:shift + b.n * (b.V + pad)].view(b.n, b.V + pad)[:, b.V:] == 5).all())
    return s, g


SHAPES = [(3, 1), (7, 2), (64, 5), (33, 15), (9, 33), (9, 257), (4, 1000), (3, 2500), (3, 4097), (6, 8191), (5, 32768),
          (3, 50001), (2, 151111), (700, 9001)]


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("n,V", SHAPES)
def test_scores(ctx, n, V, dt):
    check_scores(ctx, Batch(n, V, dt, V + n, T=1.3, masked=0.2))
    check_scores(ctx, Batch(n, V, dt, V + n + 1, T=0.7, pad=3, shift=1), ent=False, pad=5, shift=2)
    check_scores(ctx, Batch(n, V, dt, V + n + 2), logp=False)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("n,V", SHAPES)
def test_scores_of_lists(ctx, n, V, dt):
    top = min(V, 17)
    check_scores(ctx, Batch(n, V, dt, V + n, T=1.3, masked=0.2), top=top, ent=False)
    check_scores(ctx, Batch(n, V, dt, V + n + 1, pad=2), top=top, twice=True, pad=1)
    check_scores(ctx, Batch(n, V, dt, V + n + 2), logp=False, ent=False, top=1, ragged=0.0)


@pytest.mark.parametrize("V", [1500, 4000, 40_000, 200_000])
def test_scores_of_long_lists(ctx, V):
    """The longest lists, by every kernel; ids that come again."""
    check_scores(ctx, Batch(5, V, "f32", V, pad=1), top=1024, twice=True)
    b = Batch(400, V, "bf16", V + 1, out=0.3)
    check_scores(ctx, b, top=1024, ragged=0.01)
    b = Batch(3, 700, "f32", V + 2)
    check_scores(ctx, b, top=1024, twice=True)           # more places than entries


@pytest.mark.parametrize("top", [0, 9])
@pytest.mark.parametrize("n,V", [(50, 7), (50, 300), (50, 2500), (3, 9000), (1000, 9000), (5, 70_000)])
def test_scores_in_place_and_empty_rows(ctx, n, V, top):
    b = Batch(n, V, "bf16", V, masked=0.4)
    z = b.z.copy()
    z[1] = -np.inf
    b.set(z)
    s = Scores(b, top=min(top, V))
    z = b.z.copy()
    z[1] = -np.inf
    b.set(z)
    want, gt = s.want(b)
    _, g = b.grad()
    s.call(ctx, b, g)
    s.call(ctx, b, b.logits)
    ctx.sync()
    assert bool((b.logits == g).all()) and bool((g[1] == 0).all()) and bool((g[b.tok < 0] == 0).all())
    grad_close(b, g, want, gt)


def test_scores_against_differences(ctx):
    """The call's gradient against differences of the loss that the library itself computes from
    its log-probabilities, entropies and lists."""
    import torch
    n, V, K, T = 3, 40, 4, 1.2
    b = Batch(n, V, "f32", 11, T=T, out=0.0)
    ids, lp, logp, H = torch.empty((n, K), dtype=torch.int32, device="cuda"), empty(n, K), empty(n), empty(n)
    tok = cuda(b.tok)
    g, e, h = (cuda(b.rng.normal(size=s).astype(np.float32)) for s in (n, n, (n, K)))
    ctx.token_top(b.logits, ids, lp, tok, logp, H, temperature=T)
    grad = empty(n, V)
    ctx.learn_token_scores(b.logits, tok, grad, g, e, ids, h, temperature=T)
    ctx.sync()
    lists = ids.cpu().numpy()

    def loss(z):                                         # in 64 bits: differences of fp32 results are too coarse
        from oracle.token_loss import rows
        q, _, ent, _ = rows(z, b.T)
        at = np.arange(n)
        return ((q[at, b.tok] * g.cpu().numpy()).sum() + (ent * e.cpu().numpy()).sum()
                + (np.take_along_axis(q, lists, 1) * h.cpu().numpy()).sum())

    eps = 1e-5
    for i in range(n):
        for j in range(V):
            d = np.zeros_like(b.z)
            d[i, j] = eps
            diff = (loss(b.z + d) - loss(b.z - d)) / (2 * eps)
            assert abs(float(grad[i, j]) - diff) < 1e-5 * (1 + abs(diff))
    from oracle.token_loss import rows                   # and the library's values are the loss's
    q, _, ent, _ = rows(b.z, b.T)
    assert np.abs(logp.cpu().numpy() - q[np.arange(n), b.tok]).max() < 1e-5 and np.abs(H.cpu().numpy() - ent).max() < 1e-5


@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("V", [20, 300, 2500, 9000, 70_000])
def test_scores_infinite_slopes(ctx, V, top):
    b = Batch(6, V, "f32", V, masked=0.3, out=0.0)
    s = Scores(b, ent=False, top=top, ragged=0.0)
    s.g[:4] = [np.inf, -np.inf, np.nan, 1e30]
    if top:
        s.ids[4] = [-1, -1, s.ids[4, 2]]
        s.h[4, 2] = np.inf
        if s.ids[4, 2] == b.tok[4]:
            s.g[4] = 0
    _, g = b.grad()
    s.call(ctx, b, g)
    ctx.sync()
    g = g.cpu().numpy()
    p = np.exp(b.z - b.z.max(1, keepdims=True))
    def expect(i, at, sign):
        want = np.where(p[i] > 0, -sign * np.inf, 0)
        if top:                                          # a masked entry has its own slope
            for j, h in zip(s.ids[i], s.h[i]):
                if j >= 0 and p[i, j] == 0:
                    want[j] = h
        want[at] = sign * np.inf
        return want

    for i, sign in ((0, 1), (1, -1)):
        want = expect(i, b.tok[i], sign)
        np.testing.assert_array_equal(g[i], want)
    assert np.isnan(g[2]).all() and np.isfinite(g[3]).all() and np.isfinite(g[5]).all()
    if top:
        np.testing.assert_array_equal(g[4], expect(4, s.ids[4, 2], 1))


def test_scores_errors_and_refusals(ctx):
    import torch
    b = Batch(5, 900, "f32", 3, out=0.0)
    s = Scores(b, top=4, ragged=0.0)
    want, gt = s.want(b)
    s.ids[1, 2] = 900                                    # past the vocabulary: the entry is left out
    h = s.h.copy()
    h[1, 2] = 0
    b.tok[3] = 901                                       # the row is left out
    _, g = b.grad()
    s.call(ctx, b, g)
    with pytest.raises(MalibError, match="EINVAL"):
        ctx.sync()
    b.tok[3], s.ids[1, 2], s.h = -1, -1, h
    grad_close(b, g, *s.want(b))
    tok, one = cuda(b.tok.clip(0)), empty(5)
    ids, hh = torch.zeros((5, 2), dtype=torch.int32, device="cuda"), empty(5, 2)
    call = lambda *a, tokens=tok, grad=g, **k: ctx.learn_token_scores(b.logits, tokens, grad, *a, **k)  # noqa: E731
    for f in (lambda: call(one, ids=ids), lambda: call(one, top_grad=hh), lambda: call(empty(4)),
              lambda: call(one, ids=ids, top_grad=empty(5, 3)), lambda: call(one, ids=ids.long(), top_grad=hh),
              lambda: call(one, grad=g[:, :5]), lambda: call(one, ids=ids[:, :0], top_grad=hh[:, :0])):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: call(), lambda: call(one, grad=None), lambda: call(one, tokens=None), lambda: call(one.cpu()),
              lambda: call(one, temperature=-1.0),
              lambda: call(one, grad_scale=float("nan")), lambda: call(one, ids=ids.cpu(), top_grad=hh),
              lambda: call(ids=torch.zeros((5, 1025), dtype=torch.int32, device="cuda"), top_grad=empty(5, 1025))):
        with pytest.raises(MalibError, match="EINVAL"):
            f()
    ctx.learn_token_scores(b.logits[:0], tok[:0], g[:0], one[:0])
    ctx.sync()


# ---------------------------------------------------------------- dropout

class Drop:
    def __init__(self, n, d, dt, seed, pads=(0, 0, 0), shifts=(0, 0, 0)):
        import torch
        need_gpu()
        self.rng = rng = np.random.default_rng(seed)
        self.n, self.d, self.dt = n, d, dt
        self.bufs, views = [], []
        for pad, shift in zip(pads, shifts):
            buf = torch.full((n * (d + pad) + shift + 16,), 3.0, dtype=ttype(dt), device="cuda")
            self.bufs.append(buf)
            views.append(buf[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d])
        self.x, self.res, self.out = views
        for v in (self.x, self.res):
            v.copy_(torch.from_numpy(rng.normal(size=(n, d))).to(ttype(dt)))
        self.seq = rng.integers(-2 ** 50, 2 ** 50, n)
        self.step = rng.integers(0, 2 ** 31 - 1, n).astype(np.int32)
        self.pads, self.shifts = pads, shifts

    def call(self, ctx, p, seed, site, residual, x=None, out=None):
        ctx.dropout(self.x if x is None else x, self.out if out is None else out, p, seed, site, cuda(self.seq),
                    cuda(self.step), residual)

    def check(self, p, seed, site, residual, got=None, x=None, res=None):
        import torch
        x = self.x.double().cpu().numpy() if x is None else x
        if residual and res is None:
            res = self.res.double().cpu().numpy()
        want = tr.dropout(x, p, seed, site, self.seq, self.step, res)
        keep = tr.dropout_keep(self.d, p, seed, site, self.seq, self.step)
        scaled = np.where(keep, np.abs(x) * 65536 / (65536 - tr.dropout_least(p)), 0)
        # the factor's rounding, the fused one, the type's
        tol = U * scaled + (U + HALF_ULP[self.dt]) * (np.abs(want) + U * scaled) * (1 + U) + TINY[self.dt]
        got = (self.out if got is None else got).double().cpu().numpy()
        # past the type's largest value and half a step: an infinity
        most = float(torch.finfo(ttype(self.dt)).max) * (1 + HALF_ULP[self.dt] / 2)
        over = np.abs(want) >= most
        assert (got[over] == np.sign(want[over]) * np.inf).all()
        close(np.where(over, 0, got), np.where(over, 0, want), tol, "out")
        exact = 0.0 if res is None else res
        assert (got == np.broadcast_to(exact, got.shape))[~keep].all()

    def untouched(self):
        pad, shift, n, d = self.pads[2], self.shifts[2], self.n, self.d
        buf = self.bufs[2]
        assert bool((buf[:shift] == 3).all()) and bool((buf[shift + n * (d + pad):] == 3).all())
        assert bool((buf[shift:shift + n * (d + pad)].view(n, d + pad)[:, d:] == 3).all())


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (5, 8), (2, 9), (100, 15), (1000, 64), (9, 65), (4, 1000), (3, 4096), (2, 16_383),
                                 (61, 2047), (5000, 33)])
def test_dropout(ctx, n, d, dt):
    for pads, shifts in (((0, 0, 0), (0, 0, 0)), ((0, 0, 1), (0, 0, 3)), ((1, 3, 0), (1, 2, 0)), ((2, 8, 5), (7, 0, 6))):
        for p, residual in ((0.1, True), (0.5, False)):
            k = Drop(n, d, dt, n + d, pads, shifts)
            k.call(ctx, p, 0xFEDCBA9876543210, 5, k.res if residual else None)
            ctx.sync()
            k.check(p, 0xFEDCBA9876543210, 5, residual)
            k.untouched()


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("d", [64, 1001])
def test_dropout_in_place_and_ends_of_p(ctx, d, dt):
    for p in (0.0, 2.0 ** -17 * 0.99, 0.25, 1 - 2.0 ** -16):
        k = Drop(50, d, dt, d)
        x, res = k.x.double().cpu().numpy(), k.res.double().cpu().numpy()
        k.call(ctx, p, 7, 32767, k.res, out=k.x)                       # over x
        ctx.sync()
        k.check(p, 7, 32767, True, k.x, x, res)
        k = Drop(50, d, dt, d)
        k.call(ctx, p, 7, 0, k.res, out=k.res)                         # over the residual stream
        ctx.sync()
        k.check(p, 7, 0, True, k.res, x, res)


def test_dropout_shared_rows_and_odd_values(ctx):
    import torch
    k = Drop(30, 200, "bf16", 3)
    one = k.x[:1]
    k.call(ctx, 0.3, 9, 1, k.res[:1].expand(30, 200), x=one.expand(30, 200))
    ctx.sync()
    x, res = (np.repeat(v[:1].double().cpu().numpy(), 30, 0) for v in (k.x, k.res))
    k.check(0.3, 9, 1, True, x=x, res=res)
    k.x[:, ::3], k.x[:, 1::3] = np.nan, np.inf                         # dropped ones have no influence
    k.call(ctx, 0.3, 9, 1, k.res)
    ctx.sync()
    keep = tr.dropout_keep(200, 0.3, 9, 1, k.seq, k.step)
    odd = np.zeros((30, 200), bool)
    odd[:, ::3] = odd[:, 1::3] = True
    assert (~np.isfinite(k.out.float().cpu().numpy()) == (keep & odd)).all()


def test_dropout_mask_is_of_the_place(ctx):
    """Rows in another order and batch, and the gradient of a sum, see the same mask; sites, steps and
    seeds have their own; the share kept is within six standard deviations."""
    import torch
    n, d, p = 512, 256, 0.2
    k = Drop(n, d, "f32", 1)
    ones = torch.ones((n, d), device="cuda")
    seq, step = cuda(k.seq), cuda(k.step)
    out, part = torch.empty_like(ones), torch.empty((100, d), device="cuda")
    ctx.dropout(ones, out, p, 3, 2, seq, step)
    order = torch.randperm(n, device="cuda")[:100]
    ctx.dropout(ones[:100], part, p, 3, 2, seq[order].contiguous(), step[order].contiguous())
    ctx.sync()
    assert bool((part == out[order]).all())
    least = tr.dropout_least(p) / 65536
    assert abs(float((out > 0).float().mean()) - (1 - least)) < 6 * np.sqrt(least * (1 - least) / (n * d))
    for kw in (dict(seed=4, site=2), dict(seed=3, site=3)):
        other = torch.empty_like(ones)
        ctx.dropout(ones, other, p, sequence=seq, step=step, **kw)
        ctx.sync()
        same = float(((other > 0) == (out > 0)).float().mean())
        want = least ** 2 + (1 - least) ** 2
        assert abs(same - want) < 6 * np.sqrt(want * (1 - want) / (n * d))


def test_dropout_refusals(ctx):
    import torch
    k = Drop(4, 32, "f32", 1)
    seq, step = cuda(k.seq), cuda(k.step)
    ok = dict(sequence=seq, step=step)
    call = lambda x=k.x, out=k.out, p=0.1, seed=1, **kw: ctx.dropout(x, out, p, seed, **{**ok, **kw})  # noqa: E731
    for f in (lambda: call(out=k.out[:3]), lambda: call(out=k.out.half()), lambda: call(residual=k.res.half()),
              lambda: call(sequence=None), lambda: call(step=None), lambda: call(sequence=seq.int()), lambda: call(step=step[:3]),
              lambda: call(x=k.x.t(), out=k.out.t()), lambda: call(x=k.x.double(), out=k.out.double())):
        with pytest.raises(ValueError):
            f()
    wide = torch.zeros((4, 70), device="cuda")
    for f in (lambda: call(p=-0.1), lambda: call(p=1.0), lambda: call(p=float("nan")), lambda: call(site=32768),
              lambda: call(x=k.x.cpu()), lambda: call(step=step.cpu()), lambda: call(x=wide[:, :32], out=wide[:, 16:48]),
              lambda: call(residual=wide[:, :32], out=wide[:, 32:64]), lambda: call(out=k.out[:1].expand(4, 32))):
        with pytest.raises(MalibError, match="EINVAL"):
            f()
    ctx.dropout(k.x[:0], k.out[:0], 0.1, 1, sequence=seq[:0], step=step[:0])
    ctx.sync()
