"""The rollout's side of token policies in 64 bits: the most likely entries of a row, the
draw of a token, the gradient of any loss of log-probabilities and entropies, and
dropout. Plain NumPy; shares nothing with the CUDA path."""
from __future__ import annotations

import numpy as np

from . import philox
from .token_loss import entropy_slope, rows


def broken(z):
    """Rows with a NaN or +infinity."""
    return (np.isnan(z) | np.isposinf(z)).any(axis=1)


def order(z):
    """Every row's entries by falling value, the lower index first among equal ones."""
    return np.argsort(-(np.asarray(z, np.float64) + 0.0), axis=1, kind="stable")


def top(z, K, T=1.0, left=None):
    """(ids, ln p) of the first K entries, -1 and -infinity past the unmasked ones; -1 and 0
    (NaN) in rows that are left out (that are broken)."""
    n, V = z.shape
    lp, _, _, live = rows(z, T)
    bad = broken(z)
    ids = np.full((n, K), -1, np.int64)
    out = np.full((n, K), -np.inf)
    first = order(z)[:, :K]
    keep = np.take_along_axis(z, first, 1) > -np.inf
    k = first.shape[1]
    ids[:, :k] = np.where(keep, first, -1)
    out[:, :k] = np.where(keep, np.take_along_axis(lp, first, 1), -np.inf)
    left = ~live if left is None else left | ~live
    ids[left | bad], out[bad], out[left] = -1, np.nan, 0.0
    return ids, out


def rank(z, tokens):
    """1 + the entries before the row's token; 0 where there is none."""
    z = np.asarray(z, np.float64)
    at = np.maximum(tokens, 0)
    own = z[np.arange(len(z)), at][:, None]
    before = (z > own) | ((z == own) & (np.arange(z.shape[1])[None, :] < at[:, None]))
    gone = (tokens < 0) | np.isneginf(z).all(axis=1) | broken(z)
    return np.where(gone, 0, 1 + before.sum(axis=1))


def kept(z, top_k, top_p, T=1.0, slack=0.0):
    """One row's entries that may be drawn, in the order of the draw, with their probabilities.
    slack moves the border of top_p."""
    lp, p, _, _ = rows(z[None], T)
    if not top_k:
        ids = np.arange(len(z))
        return ids, p[0]
    ids = order(z[None])[0, :top_k]
    ids = ids[z[ids] > -np.inf]
    w = p[0, ids]
    cum = np.cumsum(w)
    n = 1 + int((cum[:-1] < top_p * cum[-1] + slack).sum()) if top_p < 1 else len(ids)
    return ids[:n], w[:n]


def token_uniform(seed, sequence, step, agent):
    ctr = np.empty((len(sequence), 4), np.uint32)
    s = np.asarray(sequence, np.int64).view(np.uint64)
    ctr[:, 0], ctr[:, 1] = s & np.uint64(0xFFFFFFFF), s >> np.uint64(32)
    ctr[:, 2], ctr[:, 3] = np.asarray(step, np.int32).view(np.uint32), agent
    return (philox(ctr, seed)[:, 0] >> 8) / 2.0 ** 24


def scores(z, tokens, logp_grad=None, entropy_grad=None, ids=None, top_grad=None, T=1.0):
    """The gradient at the logits of sum g ln p_token + sum e H + sum h ln p_id."""
    lp, p, H, live = rows(z, T)
    n, V = lp.shape
    live = live & (tokens >= 0)
    direct = np.zeros((n, V))
    if logp_grad is not None:
        direct[np.arange(n), np.maximum(tokens, 0)] += logp_grad
    if ids is not None:
        for i in range(n):
            have = ids[i] >= 0
            np.add.at(direct[i], ids[i][have], np.asarray(top_grad[i], np.float64)[have])
    g = direct - p * direct.sum(axis=1, keepdims=True)
    if entropy_grad is not None:
        g += np.asarray(entropy_grad, np.float64)[:, None] * entropy_slope(lp, p, H)
    return np.where(live[:, None], g / T, 0.0)


def dropout_least(p):
    """The share p in 65,536ths, to the nearest."""
    return int(np.floor(p * 65536 + 0.5))


def dropout_keep(d, p, seed, site, sequence, step):
    """[rows][d] whether an element is kept."""
    n, blocks = len(sequence), (d + 7) // 8
    s = np.repeat(np.asarray(sequence, np.int64).view(np.uint64), blocks)
    ctr = np.empty((n * blocks, 4), np.uint32)
    ctr[:, 0], ctr[:, 1] = s & np.uint64(0xFFFFFFFF), s >> np.uint64(32)
    ctr[:, 2] = np.repeat(np.asarray(step, np.int32).view(np.uint32), blocks)
    ctr[:, 3] = np.tile(np.arange(blocks, dtype=np.uint32), n) | np.uint32(2 ** 31 | site << 16)
    words = philox(ctr, seed)
    half = np.stack([words & 0xFFFF, words >> 16], axis=2).reshape(n, blocks * 8)
    return half[:, :d] >= dropout_least(p)


def dropout(x, p, seed, site, sequence, step, residual=None):
    scale = 65536.0 / (65536 - dropout_least(p))
    y = np.where(dropout_keep(x.shape[1], p, seed, site, sequence, step), np.asarray(x, np.float64) * scale, 0.0)
    return y if residual is None else y + residual
