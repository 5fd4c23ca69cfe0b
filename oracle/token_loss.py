"""Losses of token policies in 64 bits: log-probabilities, the clipped policy loss, the
preference loss and distillation from a teacher's top entries, each with its gradient
at the logits. Plain NumPy, row by row where a row has a condition of its own; shares
nothing with the CUDA path."""
from __future__ import annotations

import numpy as np


def rows(z, T=1.0):
    """ln p of every entry, p, entropy, and which rows have a distribution (some entry
    that is not -infinity). Rows without one come back as zeros."""
    y = np.asarray(z, np.float64) / T
    live = ~np.all(np.isneginf(y), axis=1)
    y = np.where(live[:, None], y, 0.0)
    with np.errstate(invalid="ignore", over="ignore"):
        d = y - y.max(axis=1, keepdims=True)
        e = np.exp(d)
        S = e.sum(axis=1, keepdims=True)
        lp = d - np.log(S)
        p = e / S
        H = -np.where(p == 0, 0.0, p * lp).sum(axis=1)
    return lp, p, H, live


def logprob(z, tokens, T=1.0):
    lp, _, H, live = rows(z, T)
    live = live & (tokens >= 0)
    i = np.arange(len(tokens))
    return np.where(live, lp[i, np.maximum(tokens, 0)], 0.0), np.where(live, H, 0.0), live


def entropy_slope(lp, p, H):
    """dH / dy_j = -p_j (ln p_j + H)."""
    with np.errstate(invalid="ignore"):
        return -np.where(p == 0, 0.0, p * (lp + H[:, None]))


def ppo(z, tokens, old, adv, weight, ref=None, lo=0.2, hi=0.2, ck=0.0, ch=0.0, T=1.0):
    """(loss, gradient, ln p, row losses, row slopes d l / d ln p, stats)."""
    lp, p, H, live = rows(z, T)
    n = len(tokens)
    logp = np.zeros(n)
    l, slope, clipped, kl = (np.zeros(n) for _ in range(4))
    grad = np.zeros_like(lp)
    dH = entropy_slope(lp, p, H)
    live = live & (tokens >= 0) & (weight != 0)
    for i in np.flatnonzero(live):
        logp[i] = lp[i, tokens[i]]
        with np.errstate(over="ignore", invalid="ignore"):
            rho = np.exp(logp[i] - old[i])
            a = 0.0 if adv[i] == 0 and np.isinf(rho) else rho * adv[i]
            b = np.clip(rho, 1 - lo, 1 + hi) * adv[i]
            clipped[i] = a > b
            l[i] = -(b if a > b else a) - (ch * H[i] if ch else 0.0)
            slope[i] = 0.0 if a > b else -a
            if ref is not None:
                r = ref[i] - logp[i]
                kl[i] = np.inf if r == np.inf else np.expm1(r) - r
                if ck:                                       # one that is only reported adds 0, however large
                    l[i] += ck * kl[i]
                    slope[i] -= ck * np.expm1(r)
            one = np.zeros(lp.shape[1])
            one[tokens[i]] = 1.0
            d = one - p[i]
            grad[i] = weight[i] / T * (np.where(d == 0, 0.0, slope[i] * d) - ch * dH[i])     # the slope may be infinite
    L = float((weight * l)[live].sum())
    M = max(1, live.sum())
    stats = np.array([live.sum(), L, clipped.sum() / M, kl.sum() / M, np.where(live, H, 0).sum() / M])
    return L, grad, logp, l, slope, stats


def pref(z, tokens, offsets, ref=None, beta=0.1, smooth=0.0, T=1.0):
    """(loss, gradient, rewards, row slopes, stats)."""
    lp, p, _, live = rows(z, T)
    live = live & (tokens >= 0)
    n, P = len(tokens), (len(offsets) - 1) // 2
    i = np.arange(n)
    gain = np.where(live, lp[i, np.maximum(tokens, 0)] - (0 if ref is None else ref), 0.0)
    R = np.array([beta * gain[offsets[s]:offsets[s + 1]].sum() for s in range(2 * P)])
    D = R[0::2] - R[1::2]
    l = (1 - smooth) * np.logaddexp(0, -D) + (smooth * np.logaddexp(0, D) if smooth else 0.0)
    dD = smooth / (1 + np.exp(-D)) - (1 - smooth) / (1 + np.exp(D))
    slope = np.zeros(n)
    for s in range(2 * P):
        slope[offsets[s]:offsets[s + 1]] = (1 - 2 * (s % 2)) * dD[s // 2] * beta / P
    slope = np.where(live, slope, 0.0)
    one = np.zeros_like(lp)
    one[i, np.maximum(tokens, 0)] = 1.0
    grad = np.where(live[:, None], slope[:, None] / T * (one - p), 0.0)
    stats = np.array([P, l.mean(), (D > 0).mean(), R[0::2].mean(), R[1::2].mean()])
    return float(l.mean()), grad, R, slope, stats


def distill(z, ids, teacher, weight, T=1.0):
    """(loss, gradient, row losses, the teacher's probabilities q [n][K], stats)."""
    lp, p, _, live = rows(z, T)
    n, K = ids.shape
    loss, q = np.zeros(n), np.zeros((n, K))
    grad = np.zeros_like(lp)
    for i in range(n):
        t = np.asarray(teacher[i], np.float64) / T
        have = (ids[i] >= 0) & ~np.isneginf(t)
        live[i] = live[i] and have.any() and weight[i] != 0
        if not live[i]:
            continue
        m = t[have].max()
        lq = t[have] - m - np.log(np.exp(t[have] - m).sum())
        qi, at = np.exp(lq), ids[i][have]
        q[i, have] = qi
        use = qi != 0
        loss[i] = T * T * (qi[use] * (lq[use] - lp[i, at[use]])).sum()
        grad[i] = p[i]
        np.subtract.at(grad[i], at, qi)
        grad[i] *= weight[i] * T
    M = max(1, live.sum())
    L = float((weight * loss)[live].sum())
    return L, grad, loss, q, np.array([live.sum(), L, loss.sum() / M])
