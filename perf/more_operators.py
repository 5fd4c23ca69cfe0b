"""A token policy's rollout step and what its learner needs beside the losses, as timed cases.

A token policy answers with entries of a vocabulary; its network, which lies
outside this framework, gives one row of logits for every position.

  top      log-probability, rank and entropy of given tokens with the `top` most
           likely entries beside them: what a rollout reports, and a teacher's
           lists for distillation
  sample   the draw of a row's token, from all entries or from the first top_k of
           which the likeliest top_p are kept, with its log-probabilities
  scores   the gradient at the logits of any loss of the log-probabilities, the
           entropies and the listed entries' log-probabilities
  dropout  dropout whose mask is a function of (seed; sequence, step, site, column),
           with the residual stream added in the same pass; its backward pass is
           the same call on the gradient

Every case is one call through ``paper_2106_07551_gb300.Context``. Sizes are this
repository's batches (4,096 environments, 25 steps, 15 actions, hidden width 64) and
generic vocabularies and widths, odd ones among them.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
MASK32 = 0xFFFFFFFF


def listed():
    return [
        # an answer's step with its alternatives shown: one row, a large vocabulary
        _case("top_one", "top", "bf16", 1, 131_072, top=20),
        # the step of a serving batch, odd vocabulary (rows that start anywhere)
        _case("top_batch", "top", "f16", 61, 50_001, top=5, temp=0.7),
        # a teacher's lists over a training batch, prompts left out
        _case("top_teacher", "top", "bf16", 8_192, 65_536, top=64, out=0.25),
        # the longest lists, 32 bits, a part of the vocabulary illegal
        _case("top_longest", "top", "f32", 333, 151_111, top=1024, masked=0.3),
        # the draw of one answer's token from the whole vocabulary
        _case("sample_one", "sample", "bf16", 1, 131_072),
        # a step of 4,096 live answers, truncated as answers are usually drawn, ended ones left out
        _case("sample_batch", "sample", "bf16", 4_096, 32_768, top_k=50, top_p=0.95, temp=0.8, out=0.1),
        # the framework's own kind of batch: 4,096 environments x 25 steps, 15 actions, illegal ones masked out
        _case("sample_actions", "sample", "f32", 102_400, 15, masked=0.3),
        # a minibatch of a loss on log-probabilities and entropies
        _case("scores_minibatch", "scores", "bf16", 4_096, 32_768, out=0.25, ent=True),
        # a loss on listed entries, 32 bits, rows padded to another stride, odd vocabulary
        _case("scores_listed", "scores", "f32", 1_111, 50_001, pad=7, top=64, ragged=0.3),
        # a step of a serving batch's hidden states with its residual stream
        _case("dropout_step", "dropout", "bf16", 61, 4_096, residual=True),
        # the framework's hidden width over 4,096 environments x 25 steps (forward, or a gradient)
        _case("dropout_hidden", "dropout", "f32", 102_400, 64),
        # the largest: hidden states of long sequences with their residual stream
        _case("dropout_largest", "dropout", "bf16", 32_768, 8_192, residual=True),
    ]


def _case(name, op, dtype, rows, width, **more):
    c = {"name": name, "op": op, "dtype": dtype, "rows": rows, "pad": 0}
    if op == "dropout":
        c.update(dim=width, p=0.1, residual=False)
    else:
        c.update(vocab=width, out=0.0, temp=1.0, masked=0.0)
    if op == "top":
        c.update(top=1)
    if op == "sample":
        c.update(top_k=0, top_p=1.0)
    if op == "scores":
        c.update(ent=False, top=0, ragged=0.0)
    c.update(more)
    return c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["top", "top", "sample", "sample", "scores", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    pad = rng.choice([0, 0, 0, 1, 8])
    if op == "dropout":
        dim = _log(rng, 16, 16_384)
        rows = _log(rng, 1, min(100_000, 1_200_000_000 // (3 * dim * BYTES[dtype])))
        c = _case("", op, dtype, rows, dim, pad=pad, p=rng.choice([0.05, 0.1, 0.5]), residual=rng.random() < 0.5)
        del c["name"]
        return c
    vocab = _log(rng, 1_000, 262_144) if rng.random() < 0.85 else _log(rng, 2, 1_000)
    rows = _log(rng, 1, min(100_000 if vocab < 1_000 else 8_192, 500_000_000 // (vocab * BYTES[dtype])))
    c = _case("", op, dtype, rows, vocab, pad=pad, out=rng.choice([0.0, 0.1, 0.4]),
              temp=rng.choice([1.0, 1.0, 0.7, 1.5]), masked=rng.choice([0.0, 0.0, 0.3]) if vocab >= 64 else 0.0)
    del c["name"]
    most = max(1, min(1024, vocab // 4, 2_000_000 // rows))
    if op == "top":
        c.update(top=_log(rng, 1, most))
    if op == "sample" and rng.random() < 0.6:
        c.update(top_k=_log(rng, 1, min(256, most)), top_p=rng.choice([1.0, 0.9, 0.95]))
    if op == "scores":
        c.update(ent=rng.random() < 0.5, top=rng.choice([0, _log(rng, 1, min(128, most))]), ragged=rng.choice([0.0, 0.3]))
    return c


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 2 + 1)
    return (_prepare_dropout if case["op"] == "dropout" else _prepare_rows)(case, int(seed), g)


def _prepare_dropout(case, seed, g):
    n, d, dt = case["rows"], case["dim"], TYPES[case["dtype"]]
    s = {"case": dict(case), "seed": 0x9E3779B97F4A7C15 * (2 * seed + 1) % 2 ** 63}
    s["x"] = torch.randn((n, d + case["pad"]), generator=g, device=DEV, dtype=dt)[:, :d]
    s["out"] = torch.empty((n, d), dtype=dt, device=DEV)
    if case["residual"]:
        s["residual"] = torch.randn((n, d), generator=g, device=DEV, dtype=dt).mul_(3)
    # positions of sequences that follow one another, as a learner packs what a rollout has played
    start = (torch.rand(n, generator=g, device=DEV) < 1 / 200).long()
    start[0] = 1
    number, at = start.cumsum(0) - 1, torch.arange(n, device=DEV)
    ids = torch.randint(0, 2 ** 40, (n,), generator=g, device=DEV)
    first = torch.where(start.bool(), at, 0).cummax(0).values
    s.update(sequence=ids[number], step=(at - first).int())
    return s


def _prepare_rows(case, seed, g):
    op, n, V, dt = case["op"], case["rows"], case["vocab"], TYPES[case["dtype"]]
    z = torch.randn((n, V + case["pad"]), generator=g, device=DEV, dtype=dt).mul_(2.5)[:, :V]
    if case["masked"]:                       # illegal entries, and padding of a vocabulary
        z.masked_fill_(torch.rand((n, V), generator=g, device=DEV) < case["masked"], -math.inf)
    tok = torch.randint(0, V, (n,), generator=g, device=DEV)
    # what a policy answers is mostly likely
    z.scatter_(1, tok[:, None], (4 + 3 * torch.randn((n, 1), generator=g, device=DEV)).to(dt))
    left = torch.rand(n, generator=g, device=DEV) < case["out"]
    s = {"case": dict(case), "logits": z, "tokens": torch.where(left, -1, tok).int()}
    f32 = lambda *shape: torch.empty(shape, device=DEV)  # noqa: E731
    i32 = lambda *shape: torch.empty(shape, device=DEV, dtype=torch.int32)  # noqa: E731
    if op == "top":
        K = case["top"]
        s.update(ids=i32(n, K), top_logp=f32(n, K), rank=i32(n), logp=f32(n), entropy=f32(n))
    if op == "sample":
        s.update(uniform=_uniform(case, z, g), token=i32(n), logp=f32(n), entropy=f32(n), draw_logp=f32(n))
    if op == "scores":
        s.update(grad=torch.empty((n, V), dtype=dt, device=DEV),
                 logp_grad=torch.randn(n, generator=g, device=DEV) / n,
                 entropy_grad=torch.randn(n, generator=g, device=DEV) * (0.1 / n) if case["ent"] else None,
                 list=None, list_grad=None)
        if case["top"]:
            K = case["top"]
            # distinct ids in no order: one of each of K parts of the vocabulary
            lo = (torch.arange(K, device=DEV) * V) // K
            ids = lo + (torch.rand((n, K), generator=g, device=DEV) * (V // K)).long()
            ids = ids.gather(1, torch.rand((n, K), generator=g, device=DEV).argsort(1))
            top = (5 + 2 * torch.randn((n, K), generator=g, device=DEV)).to(dt)
            z.scatter_(1, ids, top)
            ids[torch.rand((n, K), generator=g, device=DEV) < case["ragged"]] = -1
            s.update(list=ids.int(), list_grad=torch.randn((n, K), generator=g, device=DEV) / (n * K))
    # a loss scale for 16-bit floats of few exponents
    s["scale"] = float(2 ** math.floor(math.log2(n))) if case["dtype"] == "f16" else 1.0
    return s


def _uniform(case, z, g):
    """Random numbers whose tokens do not hang on a sum's last bits: each lies in the middle of the
    share of a token that was drawn first; rows whose kept part ends within rounding are moved."""
    n, V = z.shape
    u = torch.empty(n, device=DEV)
    for a in range(0, n, 1024):
        zb = z[a:a + 1024]
        if case["top_k"]:
            K = case["top_k"]
            for _ in range(4):
                y = zb.topk(K, 1).values.double() / case["temp"]
                w = (y - y[:, :1]).exp()
                cum = w.cumsum(1) / w.sum(1, keepdim=True)
                near = ((cum - case["top_p"]).abs() < 1e-5).any(1) & (case["top_p"] < 1.0)
                best = zb.argmax(1, keepdim=True)
                zb.scatter_(1, best, torch.where(near[:, None], zb.gather(1, best) + 0.25, zb.gather(1, best)))
            w = torch.where(cum - w / w.sum(1, keepdim=True) < case["top_p"], w, 0.0)
        else:
            y = zb.double() / case["temp"]
            w = (y - y.amax(1, keepdim=True)).exp()
        q = w / w.sum(1, keepdim=True)
        at = torch.multinomial(q.float(), 1, generator=g)
        at = torch.where(q.gather(1, at) < 2e-5, q.argmax(1, keepdim=True), at)
        u[a:a + 1024] = (q.cumsum(1).gather(1, at) - q.gather(1, at) / 2)[:, 0].float()
    return u


# ------------------------------------------------------------------ one pass

@functools.lru_cache(maxsize=1)
def _context():
    import paper_2106_07551_gb300 as mb
    return mb.Context(0, torch.cuda.current_stream(DEV))


def run(s):
    op = s["case"]["op"]
    if own:
        return {"top": _own_top, "sample": _own_sample, "scores": _own_scores, "dropout": _own_dropout}[op](s)
    return {"top": _plain_top, "sample": _plain_sample, "scores": _plain_scores, "dropout": _plain_dropout}[op](s)


def _own_top(s):
    _context().token_top(s["logits"], s["ids"], s["top_logp"], tokens=s["tokens"], logp_out=s["logp"],
                         entropy_out=s["entropy"], rank_out=s["rank"], temperature=s["case"]["temp"])
    return {k: s[k] for k in ("ids", "top_logp", "rank", "logp", "entropy")}


def _own_sample(s):
    c = s["case"]
    _context().token_sample(s["logits"], s["token"], s["logp"], s["entropy"], s["draw_logp"], tokens=s["tokens"],
                            uniform=s["uniform"], top_k=c["top_k"], top_p=c["top_p"], temperature=c["temp"])
    return {k: s[k] for k in ("token", "logp", "entropy", "draw_logp")}


def _own_scores(s):
    _context().learn_token_scores(s["logits"], s["tokens"], s["grad"], logp_grad=s["logp_grad"],
                                  entropy_grad=s["entropy_grad"], ids=s["list"], top_grad=s["list_grad"],
                                  temperature=s["case"]["temp"], grad_scale=s["scale"])
    return {"grad": s["grad"]}


def _own_dropout(s):
    _context().dropout(s["x"], s["out"], s["case"]["p"], s["seed"], site=3, sequence=s["sequence"], step=s["step"],
                       residual=s.get("residual"))
    return {"out": s["out"]}


def _log_softmax(logits, temp):
    """Log-probabilities and probabilities of every entry, in 32 bits."""
    y = logits.float() / temp
    y = y - y.amax(1, keepdim=True)
    e = y.exp()
    S = e.sum(1, keepdim=True)
    return y - S.log(), e / S


def _entropy(lp, p):
    return -torch.where(p > 0, p * lp, 0.0).sum(1)


def _order(logits):
    """Whole numbers in the entries' order: by value, the lower index first among equal ones."""
    bits = (logits.float() + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    return bits * 2 ** 24 + (2 ** 24 - 1 - torch.arange(logits.shape[1], device=logits.device))


def _plain_top(s):
    c, tok = s["case"], s["tokens"].long()
    live, at = tok >= 0, tok.clamp(min=0)[:, None]
    lp, p = _log_softmax(s["logits"], c["temp"])
    key = _order(s["logits"])
    ids = key.topk(c["top"], 1).indices
    rank = (key > key.gather(1, at)).sum(1) + 1
    top = lp.gather(1, ids)
    ids = torch.where(top == -math.inf, -1, ids)
    return {"ids": torch.where(live[:, None], ids, -1).int(), "top_logp": torch.where(live[:, None], top, 0.0),
            "rank": torch.where(live, rank, 0).int(), "logp": torch.where(live, lp.gather(1, at)[:, 0], 0.0),
            "entropy": torch.where(live, _entropy(lp, p), 0.0)}


def _plain_sample(s):
    c, live = s["case"], s["tokens"] >= 0
    lp, p = _log_softmax(s["logits"], c["temp"])
    u = s["uniform"].double()[:, None]
    if c["top_k"]:
        ids = _order(s["logits"]).topk(c["top_k"], 1).indices
        w = lp.gather(1, ids).double().exp()
        w = torch.where(w.cumsum(1) - w < c["top_p"] * w.sum(1, keepdim=True), w, 0.0)
    else:
        ids, w = None, p.double()
    cum = w.cumsum(1)
    total = cum[:, -1:]
    at = (cum <= u * total).sum(1, keepdim=True).clamp(max=w.shape[1] - 1)
    drawn = (w.gather(1, at) / total).log()[:, 0].float()
    at = at if ids is None else ids.gather(1, at)
    return {"token": torch.where(live, at[:, 0], -1).int(), "logp": torch.where(live, lp.gather(1, at)[:, 0], 0.0),
            "entropy": torch.where(live, _entropy(lp, p), 0.0), "draw_logp": torch.where(live, drawn, 0.0)}


def _plain_scores(s):
    c, tok = s["case"], s["tokens"].long()
    live, at = tok >= 0, tok.clamp(min=0)[:, None]
    lp, p = _log_softmax(s["logits"], c["temp"])
    f = torch.where(live, s["scale"] / c["temp"], 0.0)[:, None]
    total = s["logp_grad"][:, None]
    if s["list"] is not None:
        have = s["list"] >= 0
        h = torch.where(have, s["list_grad"], 0.0)
        total = total + h.sum(1, keepdim=True)
    grad = p * (f * -total)
    if s["entropy_grad"] is not None:
        H = _entropy(lp, p)[:, None]
        grad = grad - torch.where(p > 0, p * (lp + H), 0.0) * (f * s["entropy_grad"][:, None])
    if s["list"] is not None:
        grad.scatter_add_(1, s["list"].long().clamp(min=0), f * h)
    grad.scatter_add_(1, at, f * s["logp_grad"][:, None])
    return {"grad": grad.to(s["logits"].dtype)}


def _philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 of counters held in 64 bits."""
    k0, k1 = seed & MASK32, seed >> 32 & MASK32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & MASK32) ^ c1 ^ k0, b & MASK32, (a >> 32 & MASK32) ^ c3 ^ k1, a & MASK32
        k0, k1 = k0 + 0x9E3779B9 & MASK32, k1 + 0xBB67AE85 & MASK32
    return c0, c1, c2, c3


def _plain_dropout(s):
    n, d = s["x"].shape
    q, step = s["sequence"][:, None], s["step"].long()[:, None]
    block = torch.arange((d + 7) // 8, device=DEV)[None, :] + (2 ** 31 | 3 << 16)
    zero = torch.zeros_like(q + block)
    words = torch.stack(_philox((q & MASK32) + zero, (q >> 32 & MASK32) + zero, step + zero, block + zero, s["seed"]), 2)
    half = torch.stack([words & 0xFFFF, words >> 16], 3).view(n, -1)[:, :d]       # a word's low half first
    least = math.floor(s["case"]["p"] * 65536 + 0.5)
    y = torch.where(half >= least, s["x"].float() * (65536 / (65536 - least)), 0.0)
    if "residual" in s:
        y = y + s["residual"].float()
    return {"out": y.to(s["x"].dtype)}


# ------------------------------------------------------------------ work and the answers in 64 bits

def work(case):
    op, n, es = case["op"], case["rows"], BYTES[case["dtype"]]
    if op == "dropout":
        return {"bytes": n * case["dim"] * es * (3 if case["residual"] else 2) + 12 * n, "flops": 2 * n * case["dim"]}
    live, V = n * (1 - case["out"]), case["vocab"]
    read, small = live * V * es, {"top": 16, "sample": 24, "scores": 8}[op] * n
    if op == "scores":
        small += 4 * n * case["ent"]
    if op in ("top", "scores"):
        small += 8 * n * case["top"]
    return {"bytes": int(read + small + (n * V * es if op == "scores" else 0)),
            "flops": int(live * V * (10 if op == "scores" else 6))}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        return {"out": _exact_dropout(s)}
    n = case["rows"]
    one = {"top": _exact_top, "sample": _exact_sample, "scores": _exact_scores}[case["op"]]
    parts = [one(s, slice(a, min(n, a + 512))) for a in range(0, n, 512)]
    return {k: torch.cat([x[k] for x in parts]) for k in parts[0]}


def _rows64(s, b):
    y = s["logits"][b].double() / float(s["case"]["temp"])
    lse = y.logsumexp(1, keepdim=True)
    lp = y - lse
    p = lp.exp()
    H = lse[:, 0] - torch.where(p > 0, p * y, 0.0).sum(1)
    tok = s["tokens"][b].long()
    return lp, p, H, tok.clamp(min=0)[:, None], tok < 0


def _exact_top(s, b):
    lp, p, H, at, left = _rows64(s, b)
    z, K = s["logits"][b].double(), s["case"]["top"]
    ids = z.sort(dim=1, descending=True, stable=True).indices[:, :K]
    own = z.gather(1, at)
    before = torch.arange(z.shape[1], device=DEV)[None, :] < at
    rank = 1 + ((z > own) | ((z == own) & before)).sum(1)
    top = lp.gather(1, ids)
    ids = ids.masked_fill(z.gather(1, ids) == -math.inf, -1)
    return {"ids": ids.masked_fill(left[:, None], -1).int(), "top_logp": top.masked_fill(left[:, None], 0.0),
            "rank": rank.masked_fill(left, 0).int(), "logp": lp.gather(1, at)[:, 0].masked_fill(left, 0.0),
            "entropy": H.masked_fill(left, 0.0)}


def _exact_sample(s, b):
    lp, p, H, _, left = _rows64(s, b)
    c, u = s["case"], s["uniform"][b].double()[:, None]
    if c["top_k"]:
        ids = s["logits"][b].double().sort(dim=1, descending=True, stable=True).indices[:, :c["top_k"]]
        w = p.gather(1, ids)
        cum = w.cumsum(1)
        kept = 1 + (cum < c["top_p"] * cum[:, -1:]).sum(1, keepdim=True)
        mass = cum.gather(1, kept.clamp(max=c["top_k"]) - 1)
    else:
        ids, cum = torch.arange(p.shape[1], device=DEV).expand_as(p), p.cumsum(1)
        mass = cum[:, -1:]
    place = torch.searchsorted(cum, u * mass, right=True)
    token = ids.gather(1, place)
    logp = lp.gather(1, token)
    return {"token": token[:, 0].masked_fill(left, -1).int(), "logp": logp[:, 0].masked_fill(left, 0.0),
            "entropy": H.masked_fill(left, 0.0), "draw_logp": (logp - mass.log())[:, 0].masked_fill(left, 0.0)}


def _exact_scores(s, b):
    lp, p, H, at, left = _rows64(s, b)
    direct = torch.zeros_like(lp).scatter_add_(1, at, s["logp_grad"][b].double()[:, None])
    if s["list"] is not None:
        ids, h = s["list"][b].long(), s["list_grad"][b].double()
        direct.scatter_add_(1, ids.clamp(min=0), h.masked_fill(ids < 0, 0.0))
    grad = direct - p * direct.sum(1, keepdim=True)
    if s["entropy_grad"] is not None:
        grad -= s["entropy_grad"][b].double()[:, None] * torch.where(p > 0, p * (lp + H[:, None]), 0.0)
    return {"grad": (grad * (s["scale"] / float(s["case"]["temp"]))).masked_fill(left[:, None], 0.0)}


def _exact_dropout(s):
    # the generator's products in 16-bit halves, a half of a word at a time
    def product(m, x):
        lo, hi = m * (x & 0xFFFF), m * (x >> 16)
        low = lo + ((hi & 0xFFFF) << 16)
        return (hi >> 16) + (low >> 32), low & MASK32

    n, d = s["x"].shape
    out = torch.empty((n, d), device=DEV, dtype=torch.float64)
    least = int(s["case"]["p"] * 65536 + 0.5)
    for a in range(0, n, 4096):
        q, t = s["sequence"][a:a + 4096], s["step"][a:a + 4096].long()
        m, e = q.shape[0], torch.arange(d, device=DEV)
        blocks = int((d + 7) // 8)
        col = torch.arange(blocks, device=DEV)
        x = [(q % 2 ** 32)[:, None].expand(m, blocks), (q // 2 ** 32)[:, None].expand(m, blocks),
             t[:, None].expand(m, blocks), (0x80030000 + col)[None].expand(m, blocks)]
        k = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
        for _ in range(10):
            h0, l0 = product(0xD2511F53, x[0])
            h1, l1 = product(0xCD9E8D57, x[2])
            x = [h1 ^ x[1] ^ k[0], l1, h0 ^ x[3] ^ k[1], l0]
            k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
        word = torch.empty((m, d), device=DEV, dtype=torch.int64)
        for i in range(4):
            cols = e[(e % 8) // 2 == i]
            word[:, cols] = x[i][:, cols // 8]
        value = torch.where(e % 2 == 0, word % 65536, word // 65536)
        y = s["x"][a:a + m].double() * (65536 / (65536 - least)) * (value >= least)
        out[a:a + m] = y + s["residual"][a:a + m].double() if "residual" in s else y
    return out
