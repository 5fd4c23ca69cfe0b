"""Calls whose outputs lie over their inputs or over one another are refused; buffers side by side in one
allocation, and tokens drawn in place, are not. Every call here is refused by the host before a
kernel starts, or is a valid one."""
import numpy as np
import pytest

from gpu_util import context
from test_gpu_token_losses import Batch, cuda, empty
from test_gpu_token_rollout import host, ints

pytestmark = pytest.mark.gpu

from paper_2106_07551_gb300 import MalibError

N, V, K = 12, 40, 3


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


def refused(call):
    with pytest.raises(MalibError, match="EINVAL.*(overlap|apart)"):
        call()


def views(*sizes, gap=0):
    """fp32 and int32 views of one allocation, side by side."""
    import torch
    buf = torch.zeros(sum(sizes) + gap * len(sizes), device="cuda")
    at, out = 0, []
    for n in sizes:
        out.append(buf[at:at + n])
        at += n + gap
    return out


def as_int(x):
    import torch
    return x.view(torch.int32)


def test_lists(ctx):
    b = Batch(N, V, "f32", 1, out=0.3)
    tok = cuda(b.tok)
    ids, lp, logp, H, rank = ints(N, K), empty(N, K), empty(N), empty(N), ints(N)
    call = lambda i=ids, l=lp, a=logp, e=H, r=rank, t=tok, z=b.logits: ctx.token_top(z, i, l, t, a, e, r)  # noqa: E731
    first = b.logits.view(-1)                            # fp32: the logits' own memory
    for f in (lambda: call(r=tok), lambda: call(a=tok.view(logp.dtype)), lambda: call(e=logp), lambda: call(i=as_int(lp)),
              lambda: call(a=first[:N]), lambda: call(e=first[-N:]), lambda: call(l=first[5:5 + N * K].view(N, K)),
              lambda: call(r=as_int(lp.view(-1))[N * K - N:]), lambda: call(i=as_int(first[:N * K]).view(N, K))):
        refused(f)
    both = views(N + 1)[0]                               # one element in common
    refused(lambda: call(a=both[:N], e=both[1:]))
    refused(lambda: call(r=as_int(both[1:]), t=as_int(both[:N])))
    call()
    ctx.sync()
    want = [host(x).copy() for x in (ids, lp, logp, H, rank)]
    i, l, a, e, r, t = views(N * K, N * K, N, N, N, N)   # side by side
    t = as_int(t)
    t.copy_(tok)
    call(as_int(i).view(N, K), l.view(N, K), a, e, as_int(r), t)
    ctx.sync()
    for got, w in zip((as_int(i).view(N, K), l.view(N, K), a, e, as_int(r)), want):
        np.testing.assert_array_equal(host(got), w)


def test_draws(ctx):
    import torch
    b = Batch(N, V, "f32", 2, out=0.3)
    tok, u = cuda(b.tok), cuda(b.rng.random(N).astype(np.float32))
    seq, step = torch.arange(N, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    out, lp, H, dl = ints(N), empty(N), empty(N), empty(N)
    first = b.logits.view(-1)
    for k in (0, 3):
        call = lambda o=out, a=lp, e=H, d=dl, **m: ctx.token_sample(  # noqa: E731
            b.logits, o, a, e, d, **{"tokens": tok, "uniform": u, "top_k": k, **m})
        by = dict(uniform=None, sequence=seq, step=step)
        for f in (lambda: call(a=u), lambda: call(d=u), lambda: call(o=as_int(u)), lambda: call(a=tok.view(lp.dtype)),
                  lambda: call(e=lp), lambda: call(d=lp), lambda: call(o=as_int(lp)), lambda: call(a=first[:N]),
                  lambda: call(o=as_int(first[N:2 * N])), lambda: call(o=step, **by), lambda: call(a=step.view(lp.dtype), **by),
                  lambda: call(a=seq.view(torch.float32)[:N], **by), lambda: call(o=seq.view(torch.int32)[N:], **by)):
            refused(f)
        both = ints(N + 1)
        both[:N].copy_(tok)
        refused(lambda: call(o=both[1:], tokens=both[:N]))       # over the next row's token
        call()
        ctx.sync()
        want = host(out).copy()
        mine = tok.clone()
        call(o=mine, tokens=mine)
        call(a=seq.view(torch.float32)[:N])                      # not read: there are random numbers
        ctx.sync()
        np.testing.assert_array_equal(host(mine), want)
        seq.copy_(torch.arange(N, device="cuda"))


def test_scores_and_dropout(ctx):
    import torch
    b = Batch(N, V, "f32", 3, out=0.3)
    tok, g = cuda(b.tok), torch.zeros((N, V), device="cuda")
    ids, h = torch.zeros((N, K), dtype=torch.int32, device="cuda"), empty(N, K)
    flat = g.view(-1)
    call = lambda t=tok, lg=None, eg=None, i=None, hg=None: ctx.learn_token_scores(b.logits, t, g, lg, eg, i, hg)  # noqa: E731
    for f in (lambda: call(lg=flat[:N]), lambda: call(eg=flat[-N:]), lambda: call(t=as_int(flat[N:2 * N]), lg=empty(N)),
              lambda: call(i=as_int(flat[:N * K]).view(N, K), hg=h), lambda: call(i=ids, hg=flat[3:3 + N * K].view(N, K))):
        refused(f)
    call(lg=empty(N), eg=empty(N), i=ids, hg=h)
    x, out = torch.ones((N, V), device="cuda"), torch.zeros((N, V), device="cuda")
    seq, step = torch.arange(N, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    bytes_ = out.view(-1).view(torch.int64)
    refused(lambda: ctx.dropout(x, out, 0.1, 1, sequence=bytes_[2:2 + N], step=step))
    refused(lambda: ctx.dropout(x, out, 0.1, 1, sequence=seq, step=out.view(-1).view(torch.int32)[-N:]))
    ctx.dropout(x, out, 0.1, 1, sequence=seq, step=step)
    ctx.dropout(x, x, 0.1, 1, sequence=seq, step=step)
    ctx.sync()
    assert bool((out == x).all())
