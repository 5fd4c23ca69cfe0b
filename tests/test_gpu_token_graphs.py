"""Captured calls of the token losses: graphs replayed among plain calls of the same context."""
import pytest

from gpu_util import need_gpu
from test_gpu_token_losses import Batch, Distill, Ppo, Pref, cuda, empty

pytestmark = pytest.mark.gpu


class Captured:
    """One call of each loss on small inputs, its plain results, and the same calls in a graph."""

    def __init__(self, c, stream, sizes):
        import torch
        self.calls, self.outs = [], []
        for n, V, dt in sizes:
            b = Batch(n, V, dt, n + V)
            tok = cuda(b.tok)
            p, q, d = Ppo(b), Pref(b, 2), Distill(b, 5)
            dev = [cuda(x) for x in (p.old, p.adv, p.w, q.off, d.ids, d.w)]
            for kind, k in (("ppo", 5), ("pref", 5), ("distill", 3)):
                (_, g), stats = b.grad(), empty(k)
                self.outs += [g, stats]
                self.calls.append(self.call(c, kind, b, tok, dev, d.t, g, stats))
        for f in self.calls:
            f()
        c.sync()
        self.want = [x.clone() for x in self.outs]
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph, stream=stream):
            for f in self.calls:
                f()

    @staticmethod
    def call(c, kind, b, tok, dev, t, g, stats):
        old, adv, w, off, ids, wd = dev
        if kind == "ppo":
            return lambda: c.learn_token_ppo(b.logits, tok, old, adv, g, stats, weight=w, entropy_coef=0.1)
        if kind == "pref":
            return lambda: c.learn_token_pref(b.logits, tok, off, g, stats)
        return lambda: c.learn_token_distill(b.logits, ids, t, g, stats, weight=wd)

    def replay(self):
        for x in self.outs:
            x.fill_(7.0)
        self.graph.replay()

    def same(self):
        return all(bool((x == w).all()) for x, w in zip(self.outs, self.want))


# the calls' kernels: short rows and the ring, alone and in clusters
SMALL = [(9, 300, "bf16"), (5, 40_000, "bf16"), (700, 9001, "f32")]


def test_replay_after_larger_calls():
    """A larger call takes more work space; the graph's own is still its own."""
    torch = need_gpu()
    from paper_2106_07551_gb300 import Context
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), Context(0, stream) as c:
        cap = Captured(c, stream, SMALL)
        cap.replay()
        stream.synchronize()
        assert cap.same()
        others = []                                               # what was freed would be handed out again
        for n in (5_000, 50_000, 1_000_000):
            z = torch.zeros((1, 64), device="cuda").expand(n, 64)
            tok, lp = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
            stats = empty(5)
            c.token_logprob(z, tok, lp)
            c.learn_token_ppo(z, tok, lp, lp, None, stats)
            others.append(stats)
            first = stats.clone()
            cap.replay()
            c.learn_token_ppo(z, tok, lp, lp, None, stats)
            cap.replay()
            c.sync()
            assert cap.same() and bool((stats == first).all()) and float(stats[0]) == n


@pytest.mark.parametrize("warm", [0, 40])
def test_growth_during_a_capture_is_refused(warm):
    """Nothing of the refused call is in the graph, and the plain call after it is good; a call that
    needs no more than there is can be captured."""
    torch = need_gpu()
    from paper_2106_07551_gb300 import Context, MalibError
    stream = torch.cuda.Stream()
    n, V = 2000, 129
    with torch.cuda.stream(stream), Context(0, stream) as c:
        b = Batch(n, V, "f32", 3)
        p, (_, g), stats = Ppo(b), b.grad(), empty(5)
        tok, old, adv = cuda(b.tok), cuda(p.old), cuda(p.adv)
        call = lambda m: c.learn_token_ppo(b.logits[:m], tok[:m], old[:m], adv[:m], g[:m], stats)  # noqa: E731
        if warm:
            call(warm)
            c.sync()
        g.fill_(7.0)
        graph, mark = torch.cuda.CUDAGraph(), empty(1)
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(MalibError, match="ESTATE.*capture"):
                call(n)
            if warm:
                call(warm)
            mark.fill_(1.0)
        graph.replay()
        stream.synchronize()
        assert float(mark) == 1.0 and bool((g[warm:] == 7.0).all()) and (not warm or bool((g[:warm] != 7.0).all()))
        call(n)
        c.sync()
        first = (g.clone(), stats.clone())
        graph.replay()
        call(n)
        c.sync()
        assert bool((g == first[0]).all()) and bool((stats == first[1]).all()) and float(stats[0]) == (b.tok >= 0).sum()
