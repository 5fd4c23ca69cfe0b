"""The token losses through the C ABI against the 64-bit oracle: every type, vocabularies
from one entry to long odd ones, masks, strides, empty rows and lists, refusals.

Tolerances follow from the arithmetic. u = 2^-24 rounds an fp32 operation; the base-2
exponential is good to 2^-22; x = (z - m) k carries three roundings, so 2^x a relative
error of 3 ln2 u |x|; a thread adds at most V / 256 + 64 terms one after another. With X
and X2 the means of |x| and x^2 under p:
  S:     eS = 2^-22 + 2.1 u X + u (V / 256 + 64)
  ln p:  eS + 4 u (1 + |y - max y| + ln S)
  p:     2^-22 + 2.1 u |x| + eS + 4 u, relative; below 2^-126 it is 0
  H:     eS + ln2 (X (2^-22 + u (V / 256 + 64) + eS) + 2.1 u X2) + 6 u (ln S + X)
and the losses and gradients by the rules of differences from there; a gradient is
rounded once to its type."""
import threading

import numpy as np
import pytest

from gpu_util import context, need_gpu
from oracle import token_loss as tl

pytestmark = pytest.mark.gpu

from paper_2106_07551_gb300 import MalibError

U = 2.0 ** -24
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


def ttype(dt):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dt]


def f32(x):
    return float(np.float32(x))


class Batch:
    """Logits in a type (host 64-bit copy z), tokens, and a context."""

    def __init__(self, n, V, dt, seed, T=1.0, masked=0.0, out=0.2, pad=0, shift=0, sharp=2.5):
        torch = need_gpu()
        self.rng = rng = np.random.default_rng(seed)
        self.n, self.V, self.dt, self.T = n, V, dt, f32(T)
        z = rng.normal(size=(n, V)) * sharp
        if masked:
            z[rng.random((n, V)) < masked] = -np.inf
        self.live_tok = rng.integers(0, V, n).astype(np.int32)
        z[np.arange(n), self.live_tok] = 2 + rng.normal(size=n)
        self.tok = np.where(rng.random(n) < out, -1, self.live_tok).astype(np.int32)
        buf = torch.full((n * (V + pad) + shift,), 7.0, dtype=ttype(dt), device="cuda")
        self.logits = buf[shift:].view(n, V + pad)[:, :V]
        self.set(z)

    def set(self, z):
        import torch
        self.logits.copy_(torch.from_numpy(np.asarray(z, np.float64)).to(ttype(self.dt)))
        self.z = self.logits.double().cpu().numpy()

    def grad(self, pad=0, shift=0):
        import torch
        buf = torch.full((self.n * (self.V + pad) + shift + 3,), 5.0, dtype=ttype(self.dt), device="cuda")
        g = buf[shift:shift + self.n * (self.V + pad)].view(self.n, self.V + pad)[:, :self.V]
        return buf, g

    def tols(self):
        lp, p, H, live = tl.rows(self.z, self.T)
        with np.errstate(invalid="ignore"):
            x = np.where(p > 0, -(lp - lp.max(axis=1, keepdims=True)) / np.log(2), 0.0)
        lnS = -lp.max(axis=1)
        X, X2 = (p * x).sum(1), (p * x * x).sum(1)
        add = U * (self.V / 256 + 64)
        eS = 2.0 ** -22 + 2.1 * U * X + add
        d = x[np.arange(self.n), self.live_tok] * np.log(2)
        return dict(p=p, lp=lp, H=H, logp=eS + 4 * U * (1 + d + lnS),
                    ep=2.0 ** -22 + 2.1 * U * x + eS[:, None] + 4 * U,
                    eH=eS + np.log(2) * (X * (2.0 ** -22 + add + eS) + 2.1 * U * X2) + 6 * U * (lnS + X))


def cuda(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def empty(*shape):
    import torch
    return torch.full(shape, 9.0, device="cuda")


def close(got, want, tol, what):
    got = got.double().cpu().numpy() if hasattr(got, "cpu") else np.asarray(got)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.max((np.abs(got - want) / tol)[bad])))


def grad_close(b, g, want, tol, scale=1.0):
    """tol: before the rounding to the gradient's type."""
    close(g, want * scale, tol * scale + HALF_ULP[b.dt] * (np.abs(want) + tol) * scale + TINY[b.dt], "grad")


SHAPES = [(3, 1), (7, 2), (64, 5), (33, 15), (5, 33), (9, 257), (4, 1000), (3, 4097), (6, 8191), (5, 32768), (3, 50001),
          (2, 151111)]
DTYPES = ["f32", "bf16", "f16"]


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


def run_logprob(ctx, b):
    lp, H = empty(b.n), empty(b.n)
    ctx.token_logprob(b.logits, cuda(b.tok), lp, H, temperature=b.T)
    ctx.sync()
    return lp, H


def check_logprob(ctx, b):
    lp, H = run_logprob(ctx, b)
    t = b.tols()
    want, wH, live = tl.logprob(b.z, b.tok, b.T)
    close(lp, want, np.where(live, t["logp"], 0), "logp")
    close(H, wH, np.where(live, t["eH"], 0), "entropy")


class Ppo:
    def __init__(self, b, ck=0.2, ch=0.05, ref=True, weight=True, adv=None):
        rng, n = b.rng, b.n
        self.ck, self.ch, self.lo, self.hi = f32(ck), f32(ch), f32(0.2), f32(0.3)
        t = tl.rows(b.z, b.T)[0][np.arange(n), b.live_tok]
        t = np.where(np.isfinite(t), t, -1.0)
        # both clip sides and the middle, none near an edge
        self.old = (t - rng.choice([-0.6, -0.12, 0.1, 0.5], n)).astype(np.float32)
        self.adv = rng.normal(size=n).astype(np.float32) if adv is None else adv
        self.ref = (t + 0.4 * rng.normal(size=n)).astype(np.float32) if ref else None
        self.w = (rng.random(n) / n).astype(np.float32) if weight else None
        if weight and n > 3:
            self.w[3] = 0.0

    def call(self, ctx, b, g, scale=1.0, logp=None, stats=None):
        ctx.learn_token_ppo(b.logits, cuda(b.tok), cuda(self.old), cuda(self.adv), g, stats,
                            weight=None if self.w is None else cuda(self.w),
                            ref_logp=None if self.ref is None else cuda(self.ref), logp_out=logp, clip_low=self.lo,
                            clip_high=self.hi, kl_coef=self.ck, entropy_coef=self.ch, temperature=b.T, grad_scale=scale)

    def want(self, b):
        w = np.full(b.n, f32(1.0 / b.n)) if self.w is None else self.w.astype(np.float64)
        L, grad, logp, l, slope, stats = tl.ppo(b.z, b.tok, self.old.astype(np.float64), self.adv.astype(np.float64), w,
                                                None if self.ref is None else self.ref.astype(np.float64), self.lo,
                                                self.hi, self.ck, self.ch, b.T)
        t = b.tols()
        live = (b.tok >= 0) & (w != 0)
        rho = np.exp(np.minimum(logp - self.old, 50))
        e = np.zeros(b.n) if self.ref is None else np.expm1(np.minimum(self.ref - logp, 50))
        dslope = np.abs(rho * self.adv) * (t["logp"] + 8 * U) + self.ck * ((np.abs(e) + 1) * (t["logp"] + 8 * U))
        p, one = t["p"], np.zeros_like(t["p"])
        one[np.arange(b.n), np.maximum(b.tok, 0)] = 1
        dl = dslope + self.ch * t["eH"] + 8 * U * (np.abs(l) + np.abs(rho * self.adv))
        s, lpH = np.abs(slope)[:, None], np.where(p > 0, np.abs(t["lp"]) + t["H"][:, None], 0)
        gt = (dslope[:, None] * np.abs(one - p) + s * (p * t["ep"] + 4 * U * (one + p))
              + self.ch * p * (lpH * (t["ep"] + 6 * U) + t["eH"][:, None] + t["logp"][:, None]))
        gt = np.where(live[:, None], np.abs(w)[:, None] / b.T * (gt + 1e-37), 0)
        M = max(1, live.sum())
        es = np.array([0, (np.abs(w) * dl)[live].sum(), 0, (dslope / max(self.ck, 1e-9))[live].sum() / M if self.ck else 0,
                       t["eH"][live].sum() / M]) + 2 * U * np.abs(stats) + 1e-30
        return grad, gt, np.where(live, logp, 0), np.where(live, t["logp"], 0), stats, es


def check_ppo(ctx, b, **kw):
    p = Ppo(b, **kw)
    scale = 4096.0 if b.dt == "f16" else 1.0
    _, g = b.grad()
    logp, stats = empty(b.n), empty(5)
    p.call(ctx, b, g, scale, logp, stats)
    ctx.sync()
    grad, gt, wl, tlp, ws, es = p.want(b)
    grad_close(b, g, grad, gt, scale)
    close(logp, wl, tlp, "logp")
    close(stats, ws, es, "stats")
    return g


class Pref:
    def __init__(self, b, pairs, smooth=0.1, beta=0.3, ref=True, offsets=None):
        rng = b.rng
        self.beta, self.smooth, self.P = f32(beta), f32(smooth), pairs
        self.off = (np.concatenate([[0], np.sort(rng.integers(0, b.n + 1, 2 * pairs - 1)), [b.n]])
                    if offsets is None else np.asarray(offsets)).astype(np.int64)
        t = tl.rows(b.z, b.T)[0][np.arange(b.n), b.live_tok]
        self.ref = (np.where(np.isfinite(t), t, -1) + rng.normal(size=b.n)).astype(np.float32) if ref else None

    def call(self, ctx, b, g, scale=1.0, reward=None, stats=None):
        ctx.learn_token_pref(b.logits, cuda(b.tok), cuda(self.off), g, stats,
                             ref_logp=None if self.ref is None else cuda(self.ref), reward_out=reward, beta=self.beta,
                             label_smoothing=self.smooth, temperature=b.T, grad_scale=scale)

    def want(self, b):
        ref = None if self.ref is None else self.ref.astype(np.float64)
        L, grad, R, slope, stats = tl.pref(b.z, b.tok, self.off, ref, self.beta, self.smooth, b.T)
        t = b.tols()
        live = b.tok >= 0
        eR = np.array([self.beta * t["logp"][a:c][live[a:c]].sum() for a, c in zip(self.off[:-1], self.off[1:])])
        eR = eR + 2 * U * np.abs(R)
        eD = eR[0::2] + eR[1::2] + U * np.abs(R[0::2] - R[1::2])
        ds = np.zeros(b.n)                                   # the slope changes by at most 1/4 of D's change
        for s in range(2 * self.P):
            ds[self.off[s]:self.off[s + 1]] = (0.25 * eD[s // 2] + 8 * U) * self.beta / self.P
        p, one = t["p"], np.zeros_like(t["p"])
        one[np.arange(b.n), np.maximum(b.tok, 0)] = 1
        gt = ds[:, None] * np.abs(one - p) + np.abs(slope)[:, None] * (p * t["ep"] + 8 * U * (one + p))
        gt = np.where(live[:, None], (gt + 1e-37) / b.T, 0)
        m = lambda v: v.mean()  # noqa: E731
        es = np.array([0, m(eD) + 8 * U, 0, m(eR[0::2]), m(eR[1::2])]) + 2 * U * np.abs(stats)
        return grad, gt, R, eR + 1e-30, stats, es


def check_pref(ctx, b, pairs, **kw):
    p = Pref(b, pairs, **kw)
    scale = 4096.0 if b.dt == "f16" else 1.0
    _, g = b.grad()
    reward, stats = empty(2 * pairs), empty(5)
    p.call(ctx, b, g, scale, reward, stats)
    ctx.sync()
    grad, gt, R, eR, ws, es = p.want(b)
    close(reward, R, eR, "reward")
    close(stats, ws, es, "stats")
    grad_close(b, g, grad, gt, scale)


class Distill:
    def __init__(self, b, top, tdt="f32", ragged=0.3, twice=False):
        import torch
        rng = b.rng
        self.top = top
        ids = np.stack([rng.permutation(max(b.V, top))[:top] % b.V for _ in range(b.n)])
        if twice and top > 1:
            ids[:, 1] = ids[:, 0]
        ids[rng.random(ids.shape) < ragged] = -1
        if b.n > 2:
            ids[2] = -1
        z = b.z.copy()                                        # the student knows the listed entries
        for i in range(b.n):
            at = ids[i][ids[i] >= 0]
            z[i, at] = rng.normal(size=len(at)) * 2
        b.set(z)
        self.ids = ids.astype(np.int32)
        self.t = torch.from_numpy(rng.normal(size=ids.shape) * 3).to(ttype(tdt)).cuda()
        self.w = (rng.random(b.n) / b.n).astype(np.float32)

    def call(self, ctx, b, g, scale=1.0, loss=None, stats=None):
        ctx.learn_token_distill(b.logits, cuda(self.ids), self.t, g, stats, weight=cuda(self.w), loss_out=loss,
                                temperature=b.T, grad_scale=scale)

    def want(self, b):
        t64 = self.t.double().cpu().numpy()
        w = self.w.astype(np.float64)
        L, grad, loss, q, stats = tl.distill(b.z, self.ids, t64, w, b.T)
        t = b.tols()
        live = np.abs(q).sum(1) > 0
        mx = np.where(self.ids >= 0, t64, -np.inf).max(1)
        dq = np.where(self.ids >= 0, np.abs(t64 - np.where(np.isfinite(mx), mx, 0)[:, None]), 0) / b.T
        # expf to 2 ulp, four roundings of its argument, a sum of `top` terms
        eq = U * (8 + 4 * (dq + (q * dq).sum(1)[:, None]) + self.top / 32 + 40)
        at = np.maximum(self.ids, 0)
        lp = np.where(q > 0, np.take_along_axis(t["lp"], at, 1), 0.0)
        lq = np.log(np.where(q > 0, q, 1))
        elp = t["logp"][:, None] + 4 * U * np.abs(lp)
        e = (q * ((np.abs(lq) + np.abs(lp)) * (eq + 4 * U) + eq + elp)).sum(1) + U * (self.top / 32 + 8) * (
            q * (np.abs(lq) + np.abs(lp))).sum(1)
        el = np.where(live, b.T ** 2 * e, 0) + 4 * U * np.abs(loss)
        gt = t["p"] * (t["ep"] + 4 * U)
        for i in range(b.n):
            np.add.at(gt[i], at[i], q[i] * (eq[i] + 8 * U) + 4 * U * t["p"][i, at[i]])
        gt = np.where(live[:, None], w[:, None] * b.T * (gt + 1e-37), 0)
        M = max(1, live.sum())
        es = np.array([0, (w * el).sum(), el.sum() / M]) + 2 * U * np.abs(stats) + 1e-30
        return grad, gt, loss, el + 1e-30, stats, es


def check_distill(ctx, b, top, **kw):
    d = Distill(b, top, **kw)
    scale = 4096.0 if b.dt == "f16" else 1.0
    _, g = b.grad()
    loss, stats = empty(b.n), empty(3)
    d.call(ctx, b, g, scale, loss, stats)
    ctx.sync()
    grad, gt, wl, el, ws, es = d.want(b)
    close(loss, wl, el, "loss")
    close(stats, ws, es, "stats")
    grad_close(b, g, grad, gt, scale)


# ---------------------------------------------------------------- values over sizes and types

@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("n,V", SHAPES)
def test_logprob(ctx, n, V, dt):
    check_logprob(ctx, Batch(n, V, dt, V + n, T=0.8, masked=0.2))


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("n,V", SHAPES)
def test_ppo(ctx, n, V, dt):
    check_ppo(ctx, Batch(n, V, dt, V + n + 1, T=1.3, masked=0.2))


@pytest.mark.parametrize("kw", [dict(ck=0.0, ch=0.0, ref=False), dict(ch=0.0), dict(ck=0.3, ref=False, ch=0.1),
                                dict(weight=False)])
def test_ppo_terms(ctx, kw):
    check_ppo(ctx, Batch(40, 3001, "f32", 5), **kw)
    check_ppo(ctx, Batch(700, 70, "bf16", 6), **kw)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("n,V", SHAPES)
def test_pref(ctx, n, V, dt):
    check_pref(ctx, Batch(n, V, dt, V + n + 2, T=0.9, masked=0.2), 1 if n < 4 else 2)


@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("n,V", SHAPES)
def test_distill(ctx, n, V, dt):
    check_distill(ctx, Batch(n, V, dt, V + n + 3, T=1.5, masked=0.2), min(V, 17), tdt=dt)


@pytest.mark.parametrize("top,V,n,twice", [(1, 900, 6, False), (1, 40000, 3, False), (1024, 5000, 3, False),
                                           (1024, 500, 3, True), (64, 200_003, 4, True), (300, 33000, 3, True),
                                           (8, 5, 40, True)])
def test_distill_lists(ctx, top, V, n, twice):
    for tdt in DTYPES:
        check_distill(ctx, Batch(n, V, "bf16", top + V, T=0.7), top, tdt=tdt, twice=twice)


@pytest.mark.parametrize("off", [[0, 0, 30], [0, 30, 30], [0, 1, 2, 2, 30], [0, 10, 10, 10, 30], [0, 0, 0, 15, 30]])
def test_pref_empty_answers(ctx, off):
    check_pref(ctx, Batch(30, 700, "bf16", 3), (len(off) - 1) // 2, offsets=off)


def test_pref_many_pairs_and_one_long_pair(ctx):
    check_pref(ctx, Batch(4000, 129, "f32", 4), 1500)
    check_pref(ctx, Batch(5000, 64, "bf16", 5), 1)
    check_pref(ctx, Batch(300, 20000, "bf16", 5, out=0.0), 40, ref=False, smooth=0.0)


def test_single_rows_of_long_vocabularies(ctx):
    for V, dt in [(262_144, "bf16"), (262_145, "f32"), (1_000_003, "f16"), (2_000_001, "f32")]:
        b = Batch(1, V, dt, V, out=0.0)
        check_logprob(ctx, b)
        check_ppo(ctx, b)
        check_pref(ctx, b, 1)
        check_distill(ctx, b, 50, ragged=0.0)


def test_many_rows(ctx):
    check_ppo(ctx, Batch(5000, 500, "bf16", 1))
    check_logprob(ctx, Batch(20000, 15, "f32", 2, masked=0.3))
    check_ppo(ctx, Batch(20011, 5, "f32", 3, masked=0.3))
    check_distill(ctx, Batch(2500, 1000, "f16", 4), 12)


# ---------------------------------------------------------------- layouts

LAYOUTS = [(0, 1, 0, 0), (3, 0, 0, 0), (3, 5, 3, 5), (0, 0, 1, 1), (8, 0, 0, 0), (1, 2, 8, 3), (0, 3, 0, 3)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", [37, 1000, 9001])
@pytest.mark.parametrize("pad,shift,gpad,gshift", LAYOUTS)
def test_strides_alignment_and_guards(ctx, V, pad, shift, gpad, gshift, dt):
    """Logits and gradient with strides and starts of their own; what lies between and
    around the gradient's rows stays as it was."""
    b = Batch(6, V, dt, V + pad, pad=pad, shift=shift)
    p = Ppo(b)
    buf, g = b.grad(gpad, gshift)
    p.call(ctx, b, g)
    ctx.sync()
    grad, gt, *_ = p.want(b)
    grad_close(b, g, grad, gt)
    g.fill_(5.0)
    assert bool((buf == 5.0).all())
    p.call(ctx, b, g)
    first = g.clone()
    d = Pref(b, 2)
    d.call(ctx, b, g)
    ctx.sync()
    grad, gt, *_ = d.want(b)
    grad_close(b, g, grad, gt)
    p.call(ctx, b, g)
    assert bool((g == first).all())
    dist = Distill(b, 7)
    dist.call(ctx, b, g)
    ctx.sync()
    grad, gt, *_ = dist.want(b)
    grad_close(b, g, grad, gt)
    g.fill_(5.0)
    assert bool((buf == 5.0).all())


@pytest.mark.parametrize("V", [33, 5000, 33001, 140_001])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_in_place(ctx, V, dt):
    """The gradient over the logits: the same bits as into a buffer of its own."""
    b = Batch(5, V, dt, V, pad=1)
    for loss in (Ppo(b), Pref(b, 2), Distill(b, 9)):
        _, g = b.grad()
        loss.call(ctx, b, g)
        keep = b.logits.clone()
        loss.call(ctx, b, b.logits)
        ctx.sync()
        assert bool((b.logits == g).all())
        b.logits.copy_(keep)


def test_one_row_for_all(ctx):
    """Logits broadcast over the rows (stride 0)."""
    b = Batch(1, 3000, "bf16", 8, out=0.0)
    n = 50
    toks = b.rng.integers(0, 3000, n).astype(np.int32)
    wide = b.logits.expand(n, 3000)
    lp, H = empty(n), empty(n)
    ctx.token_logprob(wide, cuda(toks), lp, H)
    ctx.sync()
    want, wH, _ = tl.logprob(np.repeat(b.z, n, 0), toks)
    close(lp, want, 2e-6 * (1 + np.abs(want)), "logp")       # 2^-22 + 76 u + 4 u (1 + 25) < 2e-6 of |ln p| >= 3
    close(H, wH, 1e-5, "entropy")                            # the same, times X < 4


def test_offsets_past_32_bits(ctx):
    """More than 2^31 entries: the last rows are as good as the first."""
    torch = need_gpu()
    n, V = 16_411, 131_072
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    z = torch.zeros((n, V), dtype=torch.bfloat16, device="cuda")
    b = Batch(4, V, "bf16", 3, out=0.0)
    at = [0, 8000, n - 2, n - 1]
    z[at] = b.logits
    tok = torch.zeros(n, dtype=torch.int32, device="cuda")
    tok[at] = cuda(b.tok)
    old = torch.full((n,), -float(np.log(V)), device="cuda")
    adv = torch.ones(n, device="cuda")
    g = torch.empty_like(z)
    logp = empty(n)
    ctx.learn_token_ppo(z, tok, old, adv, g, None, logp_out=logp, clip_high=1e9, weight=adv)
    ctx.sync()
    want, _, _ = tl.logprob(b.z, b.tok)
    close(logp[at], want, b.tols()["logp"], "logp")
    assert abs(float(logp[1]) + np.log(V)) < 1e-5
    slope = -np.exp(want + np.log(V))
    one = np.zeros_like(b.z)
    one[np.arange(4), b.tok] = 1
    t = b.tols()
    ref = slope[:, None] * (one - t["p"])
    # rho's argument is rounded at 12 and old's ln V too: 2 u 12 and the error of ln p
    close(g[at], ref, np.abs(ref) * 2.0 ** -8 + np.abs(slope)[:, None] * (one + t["p"]) * 1e-5, "grad")
    assert bool((g[1, 1:] == g[1, 1]).all())
    pref_off = torch.tensor([0, n - 2, n], device="cuda")
    stats = empty(5)
    ctx.learn_token_pref(z, tok, pref_off, g, stats, beta=1e-4)
    ctx.sync()
    assert torch.isfinite(stats).all() and bool((g[n - 2:].float().abs().sum(1) > 0).all())


# ---------------------------------------------------------------- values at the edges of the types

@pytest.mark.parametrize("dt", DTYPES)
@pytest.mark.parametrize("V", [6, 2500, 40000])
def test_edge_rows(ctx, V, dt):
    """Rows of nothing but masked entries, of the type's lowest value, of that and its
    highest, with one entry left, with infinities and NaN."""
    torch = need_gpu()
    lowest = float(torch.finfo(ttype(dt)).min)
    b = Batch(9, V, dt, V, out=0.0, T=0.9)
    z = b.z.copy()
    z[0] = -np.inf
    z[1] = lowest
    z[2], z[2, 3] = lowest, -lowest
    z[3], z[3, 1] = -np.inf, 0.5
    z[4, 2] = np.inf
    z[5, 4] = np.nan
    z[6], z[6, 5] = -np.inf, np.nan
    z[7, : V // 2] = lowest
    b.tok[:] = [0, 1, 3, 1, 0, 1, 2, V - 1, 0]
    b.live_tok = b.tok
    b.set(z)
    lp, H = run_logprob(ctx, b)
    lp, H = lp.cpu().numpy(), H.cpu().numpy()
    assert lp[0] == 0 and H[0] == 0
    assert abs(lp[1] + np.log(V)) < 1e-5 and abs(H[1] - np.log(V)) < 1e-5
    assert lp[2] == 0 and H[2] == 0 and lp[3] == 0 and H[3] == 0
    assert np.isnan(lp[4:7]).all() and np.isnan(H[4:7]).all()
    ok = np.isfinite(b.z[7]).all() and np.isfinite(lp[7:]).all() and np.isfinite(H[7:]).all()
    assert ok

    def check(g):
        g = g.float().cpu().numpy()
        assert not g[0].any()                                # nothing to choose from: left out
        assert np.isnan(g[4:7]).all()
        assert np.isfinite(g[[1, 2, 3, 7, 8]]).all()
        assert not g[3, [j for j in range(V) if j != 1]].any()
        return g
    old, adv, w = np.full(9, -1, np.float32), np.ones(9, np.float32), np.ones(9, np.float32)
    _, g = b.grad()
    stats = empty(5)
    ctx.learn_token_ppo(b.logits, cuda(b.tok), cuda(old), cuda(adv), g, stats, weight=cuda(w), entropy_coef=0.1,
                        temperature=b.T, clip_high=50.0)
    ctx.sync()
    out = check(g)
    # a uniform row: p = 1 / V everywhere, its entropy term 0 up to rounding
    slope = -1.0 / V * np.e
    np.testing.assert_allclose(out[1, [2, 5]], -slope / V / b.T, rtol=2e-2,
                               atol=0.1 / V * 1e-4 + TINY[dt])
    assert float(stats[0]) == 8 and np.isnan(float(stats[1]))
    # without the rows that are NaN, the statistics are those of the others
    b.tok[4:7] = -1
    ctx.learn_token_ppo(b.logits, cuda(b.tok), cuda(old), cuda(adv), g, stats, weight=cuda(w), entropy_coef=0.1,
                        temperature=b.T, clip_high=50.0)
    ctx.sync()
    assert float(stats[0]) == 5 and bool(stats.isfinite().all()) and not g[4:7].any()
    b.tok[4:7] = [0, 1, 2]
    ctx.learn_token_pref(b.logits, cuda(b.tok), cuda(np.array([0, 4, 4, 9])[[0, 1, 3]].astype(np.int64)), g, stats)
    ctx.sync()
    assert np.isnan(g[4:7].float().cpu().numpy()).all() and not g[0].any()
    ids = np.tile(np.array([[0, 1, 2]], np.int32), (9, 1))
    ids[3], ids[2] = [1, -1, -1], [3, -1, -1]
    loss = empty(9)
    ctx.learn_token_distill(b.logits, cuda(ids), cuda(np.zeros((9, 3), np.float32)), g, None, weight=cuda(w),
                            loss_out=loss, temperature=b.T)
    ctx.sync()
    check(g)
    loss = loss.cpu().numpy()
    assert loss[0] == 0 and abs(loss[3]) < 1e-6 and abs(loss[2]) < 1e-6 and np.isnan(loss[4:7]).all()


def test_token_that_is_masked(ctx):
    """ln p = -infinity of a masked token: the formulas' values, no NaN where they have none."""
    b = Batch(2, 300, "f32", 1, out=0.0)
    z = b.z.copy()
    z[:, 7] = -np.inf
    b.set(z)
    b.tok[:] = 7
    lp, H = run_logprob(ctx, b)
    assert bool((lp == -np.inf).all()) and bool(H.isfinite().all())
    _, g = b.grad()
    stats = empty(5)
    w = np.ones(2, np.float32)
    ctx.learn_token_ppo(b.logits, cuda(b.tok), cuda(-w), cuda(np.array([1, -1], np.float32)), g, stats, weight=cuda(w))
    ctx.sync()
    # the ratio is 0: with A > 0 the unclipped term 0 is the minimum, with A < 0 the clipped one
    assert not g.any()
    np.testing.assert_allclose(float(stats[1]), 0.8, rtol=1e-6)


def test_nan_advantage_stays_in_its_row(ctx):
    b = Batch(6, 2000, "f32", 2, out=0.0)
    p = Ppo(b, adv=np.array([1, np.nan, -1, 0, 2, 1], np.float32), ref=False, ck=0, ch=0)
    _, g = b.grad()
    p.call(ctx, b, g)
    ctx.sync()
    g = g.cpu().numpy()
    assert np.isnan(g[1]).all() and np.isfinite(g[[0, 2, 3, 4, 5]]).all()


def test_teacher_edges(ctx):
    """Teacher logits of -infinity are absent; a single entry; NaN stays in its row."""
    b = Batch(4, 500, "f32", 3, out=0.0)
    ids = np.array([[3, 4, 5], [3, 4, 5], [3, -1, -1], [3, 4, 5]], np.int32)
    t = np.array([[0, -np.inf, 1], [-np.inf] * 3, [2, 0, 0], [0, np.nan, 0]], np.float32)
    _, g = b.grad()
    loss, stats = empty(4), empty(3)
    ctx.learn_token_distill(b.logits, cuda(ids), cuda(t), g, stats, loss_out=loss)
    ctx.sync()
    L, grad, wl, q, _ = tl.distill(b.z[:3], ids[:3], t[:3].astype(np.float64), np.full(3, 0.25))
    close(loss[:3], wl, 1e-5 * (1 + wl), "loss")              # ln p to 2e-6, q to 5e-6, of losses of order 10
    close(g[:3], grad, 1e-5 * np.abs(grad) + 1e-6 * 0.25, "grad")
    assert np.isnan(float(loss[3])) and float(stats[0]) == 3 and not g[1].any()


# ---------------------------------------------------------------- gradients against differences

def test_gradients_against_differences(ctx):
    """A step along a direction changes the loss by the gradient's product with it. The
    direction is of unit size and the step 2^-6: a central difference of a loss of order
    1, known to about 3e-6, over 2^-5, with h^2 / 6 of a third derivative below 1."""
    torch = need_gpu()
    b = Batch(24, 900, "f32", 11, out=0.1)
    direction = torch.from_numpy(b.rng.normal(size=b.z.shape)).float().cuda()
    losses = [Ppo(b, weight=False), Pref(b, 3), Distill(b, 20)]
    losses[2].w[:] = 1.0 / b.n
    base = b.logits.clone()
    for loss in losses:
        _, g = b.grad()
        stats = empty(3 if isinstance(loss, Distill) else 5)
        loss.call(ctx, b, g)
        d = direction / direction.norm()
        d = d + 3 * g / g.norm()                              # not only noise: along the gradient too
        d /= d.norm()
        h, vals = 2.0 ** -6, []
        for s in (1, -1):
            b.logits.copy_(base + s * h * d)
            loss.call(ctx, b, None, stats=stats)
            ctx.sync()
            vals.append(float(stats[1]))
        b.logits.copy_(base)
        diff, lin = (vals[0] - vals[1]) / (2 * h), float((g.double() * d.double()).sum())
        assert abs(diff - lin) < 3e-4, (type(loss).__name__, diff, lin)


# ---------------------------------------------------------------- calls

def test_same_bits_again_and_loss_alone(ctx):
    for n, V in [(700, 40), (90, 33001), (3, 151_111)]:
        b = Batch(n, V, "bf16", n)
        for loss, k in ((Ppo(b), 5), (Pref(b, 1), 5), (Distill(b, 5), 3)):
            outs = []
            for _ in range(3):
                _, g = b.grad()
                stats = empty(k)
                loss.call(ctx, b, g, stats=stats)
                outs.append((g, stats))
            alone = empty(k)
            loss.call(ctx, b, None, stats=alone)
            ctx.sync()
            for g, s in outs[1:]:
                assert bool((g == outs[0][0]).all()) and bool((s == outs[0][1]).all())
            close(alone, outs[0][1].double().cpu().numpy(), 1e-6 * (1 + np.abs(outs[0][1].cpu().numpy())), "loss alone")


def test_no_rows(ctx):
    torch = need_gpu()
    z = torch.empty((0, 100), device="cuda")
    none = torch.empty(0, device="cuda")
    tok = none.int()
    s5, s3 = empty(5), empty(3)
    ctx.token_logprob(z, tok, none, none)
    ctx.learn_token_ppo(z, tok, none, none, z, s5, weight=none)
    ctx.sync()
    assert s5.tolist() == [0, 0, 0, 0, 0]
    ctx.learn_token_pref(z, tok, torch.zeros(5, dtype=torch.int64, device="cuda"), z, s5)
    ctx.learn_token_distill(z, torch.empty((0, 4), dtype=torch.int32, device="cuda"), torch.empty((0, 4), device="cuda"),
                            z, s3)
    ctx.sync()
    np.testing.assert_allclose(s5.tolist(), [2, np.log(2), 0, 0, 0], rtol=1e-6)
    assert s3.tolist() == [0, 0, 0]


def test_all_rows_left_out(ctx):
    b = Batch(40, 3001, "bf16", 1, out=1.1)
    p, (_, g), stats = Ppo(b), b.grad(), empty(5)
    p.call(ctx, b, g, stats=stats)
    ctx.sync()
    assert not g.any() and stats.tolist() == [0, 0, 0, 0, 0]


def test_device_errors_are_reported_and_cleared(ctx):
    b = Batch(5, 400, "f32", 1, out=0.0)
    good, _ = run_logprob(ctx, b)
    bad = b.tok.copy()
    bad[2] = 400
    lp = empty(5)
    ctx.token_logprob(b.logits, cuda(bad), lp)
    with pytest.raises(MalibError, match="vocabulary"):
        ctx.sync()
    ctx.sync()
    keep = [0, 1, 3, 4]
    assert bool((lp[keep] == good[keep]).all()) and float(lp[2]) == 0
    ids = np.array([[0, 400]] * 5, np.int32)
    ctx.learn_token_distill(b.logits, cuda(ids), cuda(np.zeros((5, 2), np.float32)))
    with pytest.raises(MalibError, match="vocabulary"):
        ctx.sync()
    _, g = b.grad()
    for off in ([0, 3, 2, 4, 5], [1, 2, 5], [0, 2, 4], [0, 2, 9], [-3, 2, 5], [0, 7, 5], [0, 2, -1, 3, 5]):
        ctx.learn_token_pref(b.logits, cuda(b.tok), cuda(np.array(off, np.int64)), g)
        with pytest.raises(MalibError, match="offsets"):
            ctx.sync()
    again, _ = run_logprob(ctx, b)
    assert bool((again == good).all())


def test_refusals(ctx):
    torch = need_gpu()
    b = Batch(4, 64, "f32", 1)
    z, tok, v = b.logits, cuda(b.tok), torch.zeros(4, device="cuda")
    host = torch.zeros(4)
    ids, t = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    off = torch.tensor([0, 2, 4], device="cuda")
    einval = [
        lambda: ctx.token_logprob(z, tok, v, temperature=0.0),
        lambda: ctx.token_logprob(z, tok, v, temperature=-1.0),
        lambda: ctx.token_logprob(z, tok, v, temperature=float("nan")),
        lambda: ctx.token_logprob(z, tok, v, temperature=float("inf")),
        lambda: ctx.token_logprob(z, tok, v, temperature=1e-42),
        lambda: ctx.token_logprob(z, tok, host),
        lambda: ctx.token_logprob(z.cpu(), tok, v),
        lambda: ctx.token_logprob(z, tok.cpu(), v),
        lambda: ctx.token_logprob(z, None, v),
        lambda: ctx.learn_token_ppo(z, tok, host, v, z),
        lambda: ctx.learn_token_ppo(z, tok, v, None, z),
        lambda: ctx.learn_token_ppo(z, tok, v, v, z, clip_low=1.0),
        lambda: ctx.learn_token_ppo(z, tok, v, v, z, clip_high=0.0),
        lambda: ctx.learn_token_ppo(z, tok, v, v, z, kl_coef=-1.0),
        lambda: ctx.learn_token_ppo(z, tok, v, v, z, entropy_coef=float("nan")),
        lambda: ctx.learn_token_ppo(z, tok, v, v, z, grad_scale=float("inf")),
        lambda: ctx.learn_token_ppo(z, tok, v, v, z.cpu()),
        lambda: ctx.learn_token_pref(z, tok, off, z, beta=0.0),
        lambda: ctx.learn_token_pref(z, tok, off, z, label_smoothing=1.0),
        lambda: ctx.learn_token_pref(z, tok, off.cpu(), z),
        lambda: ctx.learn_token_distill(z, ids, t.cpu(), z),
        lambda: ctx.learn_token_distill(z, torch.zeros((4, 1025), dtype=torch.int32, device="cuda"),
                                        torch.zeros((4, 1025), device="cuda"), z),
        lambda: ctx.learn_token_distill(z, ids[:, :0], t[:, :0], z),
    ]
    keep = z.clone()
    for i, f in enumerate(einval):
        with pytest.raises(MalibError, match="EINVAL"):
            f()
            pytest.fail(f"call {i} was taken")
    # a gradient that overlaps the logits other than in place
    flat = torch.zeros(600, device="cuda")
    with pytest.raises(MalibError, match="overlaps"):
        ctx.learn_token_ppo(flat[:256].view(4, 64), tok, v, v, flat[64:320].view(4, 64))
    with pytest.raises(MalibError, match="overlaps"):
        ctx.learn_token_ppo(flat[:280].view(4, 70)[:, :64], tok, v, v, flat[:256].view(4, 64))
    with pytest.raises(MalibError, match="stride"):
        ctx.learn_token_ppo(z, tok, v, v, z[:1].expand(4, 64))
    for f in (lambda: ctx.token_logprob(z.double(), tok, v), lambda: ctx.token_logprob(z, tok.long(), v),
              lambda: ctx.token_logprob(z, tok[:3], v), lambda: ctx.token_logprob(z.t(), tok, v),
              lambda: ctx.token_logprob(z[0], tok, v), lambda: ctx.token_logprob(z, tok, v.double()),
              lambda: ctx.learn_token_ppo(z, tok, v, v, z.bfloat16()), lambda: ctx.learn_token_ppo(z, tok, v, v, z[:3]),
              lambda: ctx.learn_token_ppo(z, tok, v, v, z, v), lambda: ctx.learn_token_pref(z, tok, off[:2], z),
              lambda: ctx.learn_token_pref(z, tok, off.int(), z), lambda: ctx.learn_token_distill(z, ids, t[:3], z)):
        with pytest.raises(ValueError):
            f()
    ctx.sync()
    assert bool((z == keep).all())


def test_null_arguments_of_the_c_entries(ctx):
    import ctypes as C
    from paper_2106_07551_gb300 import _abi
    lib, E = _abi.load(), _abi.MALIB_EINVAL
    b = _abi.TokenBatch(None, None, 4, 64, 64, 0, 1.0)
    p, q, d = _abi.TokenPpo(), _abi.TokenPref(), _abi.TokenDistill()
    assert lib.malib_token_logprob(None, C.byref(b), None, None) == E
    assert lib.malib_token_logprob(ctx.handle, None, None, None) == E
    assert lib.malib_token_logprob(ctx.handle, C.byref(b), None, None) == E
    for f, s in ((lib.malib_learn_token_ppo, p), (lib.malib_learn_token_pref, q), (lib.malib_learn_token_distill, d)):
        assert f(None, C.byref(b), C.byref(s), None, None, None) == E
        assert f(ctx.handle, None, C.byref(s), None, None, None) == E
        assert f(ctx.handle, C.byref(b), None, None, None, None) == E
        assert f(ctx.handle, C.byref(b), C.byref(s), None, None, None) == E
    for bad in (dict(n_rows=-1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(dtype=3), dict(ld=63), dict(ld=-64),
                dict(ld=1 << 62)):
        a = dict(logits=None, tokens=None, n_rows=4, ld=64, vocab=64, dtype=0, temperature=1.0)
        a.update(bad)
        assert lib.malib_token_logprob(ctx.handle, C.byref(_abi.TokenBatch(*a.values())), None, None) == E
    ctx.sync()


def test_streams_threads_and_graphs():
    """Contexts on streams of their own from two threads, and a captured call replayed on
    new inputs, give what a single call gives."""
    torch = need_gpu()
    context().close()
    from paper_2106_07551_gb300 import Context
    errors, same = [], []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream), Context(0, stream) as c:
                b = Batch(64 + i, 6001 + i, "bf16", i)
                p, stats = Ppo(b), empty(5)
                _, g = b.grad()
                p.call(c, b, g, stats=stats)
                c.sync()
                first = (g.clone(), stats.clone())
                for _ in range(200):
                    p.call(c, b, g, stats=stats)
                c.sync()
                same.append(bool((g == first[0]).all()) and bool((stats == first[1]).all()))
        except Exception as e:                           # noqa: BLE001 (reported by the main thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert same == [True, True]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), Context(0, stream) as c:
        b = Batch(33, 5000, "f16", 4)
        d = Pref(b, 3)
        tok, off, ref = cuda(b.tok), cuda(d.off), cuda(d.ref)
        _, g = b.grad()
        stats = empty(5)
        call = lambda out: c.learn_token_pref(b.logits, tok, off, out, stats, ref_logp=ref)  # noqa: E731
        call(g)
        c.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(g)
        b.set(b.z[::-1].copy())
        graph.replay()
        stream.synchronize()
        got, gs = g.clone(), stats.clone()
        call(g)
        c.sync()
        assert bool((got == g).all()) and bool((gs == stats).all())


# ---------------------------------------------------------------- more rows than CTAs: rows are claimed

LOADED = [(1300, 4600, "bf16"), (700, 9001, "bf16"), (900, 5003, "f32"), (620, 17000, "f16"), (330, 60_001, "bf16"),
          (320, 31_000, "f32"), (170, 120_003, "bf16"), (160, 70_001, "f32")]


@pytest.mark.parametrize("n,V,dt", LOADED)
def test_more_rows_than_the_device_holds(ctx, n, V, dt):
    """Rows of every length class that CTAs claim one after another, with rows left out
    among them and masked entries; also in place, and the same bits each time."""
    b = Batch(n, V, dt, n + V, T=0.9, masked=0.1, out=0.3)
    check_ppo(ctx, b)
    check_logprob(ctx, b)
    scale = 4096.0 if dt == "f16" else 1.0
    p, first = Ppo(b), None
    for _ in range(3):
        _, g = b.grad(pad=1)                                  # rows aligned differently from the logits'
        stats = empty(5)
        p.call(ctx, b, g, scale, stats=stats)
        ctx.sync()
        first = first or (g, stats)
        assert bool((g == first[0]).all()) and bool((stats == first[1]).all())
    keep = b.logits.clone()
    p.call(ctx, b, b.logits, scale)
    ctx.sync()
    assert bool((b.logits == first[0]).all())
    b.logits.copy_(keep)
    check_pref(ctx, b, 3)


@pytest.mark.parametrize("n,V,dt", LOADED[::2])
def test_distill_more_rows_than_the_device_holds(ctx, n, V, dt):
    b = Batch(n, V, dt, n + V, T=1.2, out=0.0)
    check_distill(ctx, b, 40, tdt=dt)
    d, (_, g) = Distill(b, 30, twice=True), b.grad()
    outs = []
    for target in (g, b.logits.clone(), None):
        stats, loss = empty(3), empty(n)
        d.call(ctx, b, target, loss=loss, stats=stats)
        ctx.sync()
        outs.append((stats, loss))
    for s, l in outs[1:]:
        assert bool((s[:1] == outs[0][0][:1]).all())
        close(l, outs[0][1].double().cpu().numpy(), 2e-5 * (1 + outs[0][1].abs().double().cpu().numpy()), "loss")


def test_many_calls_in_a_row_leave_nothing_behind(ctx):
    """Calls of different lengths one after another on one context: counters and work
    space start as they did."""
    cases = [Batch(n, V, "bf16", n + V) for n, V in [(700, 9001), (3, 40000), (2000, 60), (50, 300), (1, 200_000), (900, 12)]]
    losses = [(b, Ppo(b)) for b in cases]
    first = []
    for rep in range(4):
        for i, (b, p) in enumerate(losses):
            _, g = b.grad()
            stats = empty(5)
            p.call(ctx, b, g, stats=stats)
            if rep == 0:
                first.append((g, stats))
            else:
                assert bool((g == first[i][0]).all()) and bool((stats == first[i][1]).all())
    ctx.sync()


@pytest.mark.parametrize("n,V,dt", [(156, 240_003, "bf16"), (153, 121_001, "f32"), (154, 240_050, "f32")])
def test_very_long_rows_one_after_another(ctx, n, V, dt):
    """More rows of 480 KB and more than the device has SMs: clusters take several each."""
    b = Batch(n, V, dt, n + V, T=1.1, masked=0.05, out=0.2)
    check_ppo(ctx, b)
    p, (_, g), stats = Ppo(b), b.grad(pad=3), empty(5)
    p.call(ctx, b, g, stats=stats)
    ctx.sync()
    p.call(ctx, b, b.logits)
    ctx.sync()
    assert bool((b.logits == g).all())


def test_distill_very_long_rows(ctx):
    b = Batch(160, 122_003, "f32", 5, T=1.3)
    check_distill(ctx, b, 1024)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("vectors", [64, 128, 256, 512, 768])
@pytest.mark.parametrize("past", [-1, 0, 1])
def test_lengths_where_the_kernel_changes(ctx, dt, vectors, past):
    """Rows of as many 16-byte vectors as one kernel takes, one entry less and one more,
    aligned and not, gradients aligned alike and differently."""
    W = 4 if dt == "f32" else 8
    for V, pad in ((vectors * W + past, 0), (vectors * W - W + 1 + past, 1)):
        b = Batch(41, V, dt, V, T=0.8, masked=0.1, out=0.2, pad=pad)
        check_logprob(ctx, b)
        check_ppo(ctx, b)
        check_pref(ctx, b, 4)
        p, (_, g) = Ppo(b), b.grad(pad=3)
        p.call(ctx, b, g)
        ctx.sync()
        _, h = b.grad()
        p.call(ctx, b, h)
        ctx.sync()
        assert bool((g == h).all())
        check_distill(ctx, Batch(41, V, dt, V + 1, T=1.5, out=0.0, pad=pad), 33, tdt=dt)
