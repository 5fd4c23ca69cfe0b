"""The losses of token policies, as timed cases.

A token policy answers with entries of a vocabulary; its network, which lies
outside this framework, gives one row of logits for every position. The learner
turns such rows into a loss and the gradient at the logits:

  logprob   log-probabilities and entropies of given tokens: what a rollout
            records, one row per live sequence, and the reference's pass over
            a whole batch
  ppo       the clipped surrogate with a KL term and an entropy term
  pref      the preference loss of (chosen, rejected) sequence pairs
  distill   distillation from a teacher's top logits

Every case is one call through ``paper_2106_07551_gb300.Context``. Sizes are this
repository's batches (episodes of 25 steps, 4,096 environments, 15 actions) and
generic vocabularies, odd ones among them.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
CLIP_LOW, CLIP_HIGH, BETA, SMOOTH = 0.2, 0.25, 0.1, 0.05


def listed():
    return [
        # a rollout's step of one sequence: log-probability and entropy of the drawn token, a single row
        _case("logprob_one", "logprob", "bf16", 1, 131_072),
        # the step of a serving batch, one row per live sequence, odd vocabulary (rows that start anywhere)
        _case("logprob_batch", "logprob", "f16", 61, 50_001, temp=0.7),
        # the reference policy's pass over a training batch with its prompt tokens left out
        _case("logprob_reference", "logprob", "bf16", 8_192, 65_536, out=0.25),
        # one episode of 25 steps
        _case("ppo_episode", "ppo", "bf16", 25, 32_768),
        # an ordinary minibatch with every term: clipped surrogate, KL to a reference, entropy, temperature
        _case("ppo_minibatch", "ppo", "bf16", 4_096, 32_768, out=0.25, kl=0.05, ent=0.01, temp=0.8),
        # the largest: long sequences over a large vocabulary
        _case("ppo_largest", "ppo", "bf16", 16_384, 131_072, out=0.1, kl=0.05),
        # 32-bit logits in rows padded to another stride, odd vocabulary
        _case("ppo_f32_padded", "ppo", "f32", 1_111, 50_001, pad=7, ent=0.01),
        # the framework's own kind of batch: 4,096 environments x 25 steps, 15 actions, illegal ones masked out
        _case("ppo_actions", "ppo", "f32", 102_400, 15, ent=0.01, masked=0.3),
        # preference pairs: a few short answers
        _case("pref_short", "pref", "bf16", 333, 32_768, pairs=4, out=0.2),
        # preference pairs: long answers
        _case("pref_long", "pref", "bf16", 8_192, 65_536, pairs=12, out=0.2),
        # distillation of a training batch from the teacher's top 64
        _case("distill_batch", "distill", "bf16", 4_096, 50_000, top=64, temp=2.0),
        # distillation in 32 bits, odd vocabulary, ragged lists
        _case("distill_f32_ragged", "distill", "f32", 333, 151_111, top=20, ragged=0.3),
    ]


def _case(name, op, dtype, rows, vocab, **more):
    c = {"name": name, "op": op, "dtype": dtype, "rows": rows, "vocab": vocab, "pad": 0, "out": 0.0, "temp": 1.0,
         "masked": 0.0}
    if op == "ppo":
        c.update(kl=0.0, ent=0.0)
    if op == "pref":
        c.update(pairs=1)
    if op == "distill":
        c.update(top=1, ragged=0.0)
    c.update(more)
    return c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprob", "ppo", "ppo", "pref", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    vocab = _log(rng, 1_000, 262_144) if rng.random() < 0.85 else _log(rng, 2, 1_000)
    most = min(100_000 if vocab < 1_000 else 16_384, 3_000_000_000 // (vocab * BYTES[dtype]))
    rows = _log(rng, 2 if op == "pref" else 1, most)
    c = _case("", op, dtype, rows, vocab, pad=rng.choice([0, 0, 0, 1, 8]), out=rng.choice([0.0, 0.1, 0.4]),
              temp=rng.choice([1.0, 1.0, 0.7, 1.5]), masked=rng.choice([0.0, 0.0, 0.3]))
    del c["name"]
    if op == "ppo":
        c.update(kl=rng.choice([0.0, 0.05]), ent=rng.choice([0.0, 0.01]))
    if op == "pref":
        c.update(pairs=_log(rng, 1, max(1, min(64, rows // 2))))
    if op == "distill":
        c.update(top=_log(rng, 1, max(1, min(128, vocab // 2))), ragged=rng.choice([0.0, 0.3]))
    return c


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 2 + 1)
    op, n, V, dt = case["op"], case["rows"], case["vocab"], TYPES[case["dtype"]]
    z = torch.randn((n, V + case["pad"]), generator=g, device=DEV, dtype=dt).mul_(2.5)[:, :V]
    if case["masked"]:                       # illegal entries, and padding of a vocabulary
        z.masked_fill_(torch.rand((n, V), generator=g, device=DEV) < case["masked"], -math.inf)
    tok = torch.randint(0, V, (n,), generator=g, device=DEV)
    # what a policy answers is mostly likely
    z.scatter_(1, tok[:, None], (4 + 3 * torch.randn((n, 1), generator=g, device=DEV)).to(dt))
    left = torch.rand(n, generator=g, device=DEV) < case["out"]
    s = {"case": dict(case), "logits": z}
    if op != "logprob":
        s["grad"] = torch.empty((n, V), dtype=dt, device=DEV)
    if op in ("logprob", "ppo", "pref"):
        logp = (z.gather(1, tok[:, None])[:, 0].float() / case["temp"]
                - torch.logsumexp(z.float() / case["temp"], 1))
    if op == "pref":
        # 2 x pairs sequences of random lengths over the rows; the first part of each is its prompt
        S = 2 * case["pairs"]
        cut = torch.randint(0, n + 1, (S - 1,), generator=g, device=DEV).sort().values
        off = torch.cat([cut.new_zeros(1), cut, cut.new_full((1,), n)])
        seg = torch.searchsorted(off[1:], torch.arange(n, device=DEV), right=True).clamp_(max=S - 1)
        pos = torch.arange(n, device=DEV) - off[seg]
        left = pos < case["out"] * (off[seg + 1] - off[seg])
        s.update(offsets=off, ref=logp + 0.3 * torch.randn(n, generator=g, device=DEV),
                 reward=torch.empty(S, device=DEV), stats=torch.empty(5, device=DEV))
    if op == "ppo":
        # the policy moved a little since it acted; ratios within rounding of a clip edge are moved off it
        lr = 0.15 * torch.randn(n, generator=g, device=DEV)
        for edge in (math.log(1 - CLIP_LOW), math.log(1 + CLIP_HIGH)):
            lr = torch.where((lr - edge).abs() < 2e-3, lr + 5e-3, lr)
        s.update(old=logp - lr, adv=torch.randn(n, generator=g, device=DEV),
                 ref=logp + 0.2 * torch.randn(n, generator=g, device=DEV) if case["kl"] else None,
                 logp=torch.empty(n, device=DEV), stats=torch.empty(5, device=DEV))
    if op == "distill":
        K = case["top"]
        # distinct ids in no order: one of each of K parts of the vocabulary
        lo = (torch.arange(K, device=DEV) * V) // K
        ids = lo + (torch.rand((n, K), generator=g, device=DEV) * (V // K)).long()
        ids = ids.gather(1, torch.rand((n, K), generator=g, device=DEV).argsort(1))
        top = (6 + 2 * torch.randn((n, K), generator=g, device=DEV)).sort(1, descending=True).values
        z.scatter_(1, ids, (0.8 * top + torch.randn((n, K), generator=g, device=DEV)).to(dt))
        ids[torch.rand((n, K), generator=g, device=DEV) < case["ragged"]] = -1
        ids[left] = -1
        s.update(ids=ids.int(), top=top.to(dt), loss=torch.empty(n, device=DEV), stats=torch.empty(3, device=DEV))
    else:
        s["tokens"] = torch.where(left, -1, tok).int()
    if op in ("ppo", "distill"):
        s["weight"] = torch.full((n,), 1.0 / n, device=DEV)
    if op == "logprob":
        s.update(logp=torch.empty(n, device=DEV), entropy=torch.empty(n, device=DEV))
    # a loss scale for 16-bit floats of few exponents
    s["scale"] = float(2 ** math.floor(math.log2(n))) if case["dtype"] == "f16" else 1.0
    return s


# ------------------------------------------------------------------ one pass

@functools.lru_cache(maxsize=1)
def _context():
    import paper_2106_07551_gb300 as mb
    return mb.Context(0, torch.cuda.current_stream(DEV))


def run(s):
    op = s["case"]["op"]
    if own:
        return {"logprob": _own_logprob, "ppo": _own_ppo, "pref": _own_pref, "distill": _own_distill}[op](s)
    return {"logprob": _plain_logprob, "ppo": _plain_ppo, "pref": _plain_pref, "distill": _plain_distill}[op](s)


def _own_logprob(s):
    _context().token_logprob(s["logits"], s["tokens"], s["logp"], s["entropy"], temperature=s["case"]["temp"])
    return {"logp": s["logp"], "entropy": s["entropy"]}


def _own_ppo(s):
    c = s["case"]
    _context().learn_token_ppo(s["logits"], s["tokens"], s["old"], s["adv"], s["grad"], s["stats"], weight=s["weight"],
                               ref_logp=s["ref"], logp_out=s["logp"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                               kl_coef=c["kl"], entropy_coef=c["ent"], temperature=c["temp"], grad_scale=s["scale"])
    return {"grad": s["grad"], "logp": s["logp"], "stats": s["stats"]}


def _own_pref(s):
    c = s["case"]
    _context().learn_token_pref(s["logits"], s["tokens"], s["offsets"], s["grad"], s["stats"], ref_logp=s["ref"],
                                reward_out=s["reward"], beta=BETA, label_smoothing=SMOOTH, temperature=c["temp"],
                                grad_scale=s["scale"])
    return {"grad": s["grad"], "reward": s["reward"], "stats": s["stats"]}


def _own_distill(s):
    c = s["case"]
    _context().learn_token_distill(s["logits"], s["ids"], s["top"], s["grad"], s["stats"], weight=s["weight"],
                                   loss_out=s["loss"], temperature=c["temp"], grad_scale=s["scale"])
    return {"grad": s["grad"], "loss": s["loss"], "stats": s["stats"]}


def _log_softmax(logits, temp):
    """Log-probabilities and probabilities of every entry, in 32 bits."""
    y = logits.float() / temp
    y = y - y.amax(1, keepdim=True)
    e = y.exp()
    S = e.sum(1, keepdim=True)
    return y - S.log(), e / S


def _entropy(lp, p):
    return -torch.where(p > 0, p * lp, 0.0).sum(1)


def _plain_logprob(s):
    tok, c = s["tokens"].long(), s["case"]
    live = tok >= 0
    lp, p = _log_softmax(s["logits"], c["temp"])
    logp = lp.gather(1, tok.clamp(min=0)[:, None])[:, 0]
    return {"logp": torch.where(live, logp, 0.0), "entropy": torch.where(live, _entropy(lp, p), 0.0)}


def _plain_ppo(s):
    tok, c = s["tokens"].long(), s["case"]
    live, at = tok >= 0, tok.clamp(min=0)[:, None]
    lp, p = _log_softmax(s["logits"], c["temp"])
    logp = lp.gather(1, at)[:, 0]
    H = _entropy(lp, p)
    rho = (logp - s["old"]).exp()
    free, cut = rho * s["adv"], rho.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * s["adv"]
    clipped = free > cut
    loss = -torch.where(clipped, cut, free) - c["ent"] * H
    slope = torch.where(clipped, 0.0, -free)
    kl = torch.zeros_like(loss)
    if s["ref"] is not None:
        r = s["ref"] - logp
        kl = r.exp() - r - 1
        loss = loss + c["kl"] * kl
        slope = slope + c["kl"] * (1 - r.exp())
    w = torch.where(live, s["weight"], 0.0)
    out = w * (s["scale"] / c["temp"])
    grad = p * (out * -slope)[:, None]
    if c["ent"]:
        grad = grad + p * torch.where(p > 0, lp + H[:, None], 0.0) * (out * c["ent"])[:, None]
    grad.scatter_add_(1, at, (out * slope)[:, None])
    M = live.sum()
    mean = lambda x: torch.where(live, x, 0.0).sum() / M.clamp(min=1)  # noqa: E731
    stats = torch.stack([M.float(), torch.where(live, w * loss, 0.0).sum(), mean(clipped.float()), mean(kl), mean(H)])
    return {"grad": grad.to(s["logits"].dtype), "logp": torch.where(live, logp, 0.0), "stats": stats}


def _plain_pref(s):
    tok, off, c = s["tokens"].long(), s["offsets"], s["case"]
    live, at = tok >= 0, tok.clamp(min=0)[:, None]
    lp, p = _log_softmax(s["logits"], c["temp"])
    n, S = tok.shape[0], off.shape[0] - 1
    seg = torch.searchsorted(off[1:], torch.arange(n, device=tok.device), right=True)
    gain = torch.where(live, lp.gather(1, at)[:, 0] - s["ref"], 0.0)
    reward = BETA * torch.zeros(S, device=tok.device).index_add_(0, seg, gain)
    d = reward[0::2] - reward[1::2]
    soft = lambda x: x.clamp(min=0) + (1 + (-x.abs()).exp()).log()  # noqa: E731, ln(1 + e^x)
    loss = (1 - SMOOTH) * soft(-d) + SMOOTH * soft(d)
    slope = (1 / (1 + (-d).exp()) - (1 - SMOOTH)) * (BETA * s["scale"] / (c["temp"] * (S // 2)))
    row = torch.where(live, torch.stack([slope, -slope], 1).reshape(-1)[seg], 0.0)
    grad = p * -row[:, None]
    grad.scatter_add_(1, at, row[:, None])
    stats = torch.stack([loss.new_tensor(S // 2), loss.mean(), (d > 0).float().mean(), reward[0::2].mean(),
                         reward[1::2].mean()])
    return {"grad": grad.to(s["logits"].dtype), "reward": reward, "stats": stats}


def _plain_distill(s):
    ids, c = s["ids"].long(), s["case"]
    have, at, T = ids >= 0, ids.clamp(min=0), c["temp"]
    live = have.any(1)
    t = torch.where(have, s["top"].float() / T, -math.inf)
    t = t - torch.where(live, t.amax(1), 0.0)[:, None]
    S = t.exp().sum(1, keepdim=True).clamp(min=1e-30)
    q = t.exp() / S
    lp, p = _log_softmax(s["logits"], T)
    loss = T * T * torch.where(q > 0, q * (t - S.log() - lp.gather(1, at)), 0.0).sum(1)
    w = torch.where(live, s["weight"], 0.0)
    out = (w * (s["scale"] * T))[:, None]
    grad = (p * out).scatter_add_(1, at, -q * out)
    M = live.sum()
    stats = torch.stack([M.float(), (w * loss).sum(), loss.sum() / M.clamp(min=1)])
    return {"grad": grad.to(s["logits"].dtype), "loss": loss, "stats": stats}


# ------------------------------------------------------------------ work and the answers in 64 bits

def work(case):
    op, n, V, es = case["op"], case["rows"], case["vocab"], BYTES[case["dtype"]]
    live = n if op == "distill" and not case["out"] else n * (1 - case["out"])
    read, write = live * V * es, 0 if op == "logprob" else n * V * es
    small = {"logprob": 12, "ppo": 20, "pref": 8, "distill": 8}[op] * n
    if op == "distill":
        small += n * case["top"] * (4 + es)
    return {"bytes": int(read + write + small), "flops": int(live * V * (6 if op == "logprob" else 10))}


def exact(case, seed):
    s = prepare(case, seed)
    op, n, T = case["op"], case["rows"], float(case["temp"])
    f64 = lambda k: s[k].double()  # noqa: E731
    blocks = [slice(a, min(n, a + 1024)) for a in range(0, n, 1024)]
    lse, H = torch.empty(n, device=DEV, dtype=torch.float64), torch.empty(n, device=DEV, dtype=torch.float64)
    for b in blocks:
        y = s["logits"][b].double() / T
        lse[b] = y.logsumexp(1)
        p = (y - lse[b, None]).exp()
        H[b] = lse[b] - torch.where(p > 0, p * y, 0.0).sum(1)
    if op == "distill":
        ids = s["ids"].long()
        t = (f64("top") / T).masked_fill(ids < 0, -math.inf)
        live = (ids >= 0).any(1)
        lq = t - t.masked_fill(~live[:, None], 0.0).logsumexp(1)[:, None]
        q = torch.where(ids >= 0, lq.exp(), 0.0)
        lpk = s["logits"].gather(1, ids.clamp(min=0)).double() / T - lse[:, None]
        loss = T * T * torch.where(q > 0, q * (lq - lpk), 0.0).sum(1)
        k = torch.where(live, f64("weight"), 0.0) * s["scale"] * T
        grad = torch.zeros((n, case["vocab"]), device=DEV, dtype=torch.float64)
        for b in blocks:
            grad[b] = (s["logits"][b].double() / T - lse[b, None]).exp()
            grad[b].scatter_add_(1, ids[b].clamp(min=0), -q[b])
            grad[b] *= k[b, None]
        M = int(live.sum())
        stats = [M, float((f64("weight") * loss).sum()), float(loss.sum()) / max(1, M)]
        return {"grad": grad, "loss": loss, "stats": torch.tensor(stats, dtype=torch.float64)}
    tok = s["tokens"].long()
    live = tok >= 0
    at = tok.clamp(min=0)
    logp = torch.where(live, s["logits"].gather(1, at[:, None])[:, 0].double() / T - lse, 0.0)
    if op == "logprob":
        return {"logp": logp, "entropy": torch.where(live, H, 0.0)}
    h = torch.zeros_like(logp)
    if op == "ppo":
        A, ratio = f64("adv"), (logp - f64("old")).exp()
        out = ((A > 0) & (ratio > 1 + CLIP_HIGH)) | ((A < 0) & (ratio < 1 - CLIP_LOW))
        loss = -A * torch.where(out, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH), ratio) - case["ent"] * H
        c = torch.where(out, 0.0, -A * ratio)
        kl = torch.zeros_like(loss)
        if s["ref"] is not None:
            kl = (f64("ref") - logp).expm1() - (f64("ref") - logp)
            loss = loss + case["kl"] * kl
            c = c - case["kl"] * (f64("ref") - logp).expm1()
        w = torch.where(live, f64("weight"), 0.0)
        c, h = c * w * s["scale"] / T, case["ent"] * w * s["scale"] / T
        M = int(live.sum())
        stats = [M, float((w * loss).sum())] + [float(x[live].double().sum()) / max(1, M) for x in (out, kl, H)]
        rest = {"logp": logp}
    else:
        off = s["offsets"].tolist()
        gain = torch.where(live, logp - f64("ref"), 0.0)
        reward = torch.stack([gain[a:b].sum() for a, b in zip(off[:-1], off[1:])]) * BETA
        d = reward[0::2] - reward[1::2]
        loss = -(1 - SMOOTH) * torch.nn.functional.logsigmoid(d) - SMOOTH * torch.nn.functional.logsigmoid(-d)
        slope = (SMOOTH * d.sigmoid() - (1 - SMOOTH) * (-d).sigmoid()) * BETA * s["scale"] / T / len(d)
        c = torch.zeros_like(logp)
        for i in range(len(off) - 1):
            c[off[i]:off[i + 1]] = slope[i // 2] * (1 - 2 * (i % 2))
        c = torch.where(live, c, 0.0)
        stats = [len(d), float(loss.mean()), float((d > 0).double().mean()), float(reward[0::2].mean()),
                 float(reward[1::2].mean())]
        rest = {"reward": reward}
    grad = torch.empty((n, case["vocab"]), device=DEV, dtype=torch.float64)
    for b in blocks:
        lp = s["logits"][b].double() / T - lse[b, None]
        p = lp.exp()
        grad[b] = -c[b, None] * p + h[b, None] * torch.where(p > 0, p * (lp + H[b, None]), 0.0)
        grad[b].scatter_add_(1, at[b, None], c[b, None])
    return {"grad": grad, "stats": torch.tensor(stats, dtype=torch.float64), **rest}
