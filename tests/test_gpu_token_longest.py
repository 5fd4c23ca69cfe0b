"""Rows of the longest vocabulary, 2^24 entries: the sums of a row are as good as a short one's."""
import numpy as np
import pytest

from gpu_util import context, need_gpu
from test_gpu_token_losses import U, ttype

pytestmark = pytest.mark.gpu

V = 1 << 24
# One after another, 64 entries of a stage are added at most, in two sums, then the warps' and the
# CTAs'; the sums of stages carry their rounding errors along. So ln p and H are as for any row,
# with 64 terms in place of a thread's share of the row.
ADD = 64 * U


class Row:
    """Every entry at `low` but the first 2^14 of each 2^18, at 0, so that every thread has a few that
    are larger; and the row's statistics in 64 bits, with the tolerances of ln p and H."""

    def __init__(self, dt, low):
        torch = need_gpu()
        self.z = torch.full((1, V), low, dtype=ttype(dt), device="cuda")
        self.z.view(64, -1)[:, :1 << 14] = 0
        self.low = float(self.z[0, -1])
        ones, rest = 64 << 14, V - (64 << 14)
        S = ones + rest * np.exp(self.low)
        self.lnS, p = np.log(S), np.exp(self.low) / S
        self.H = self.lnS - rest * p * self.low
        x = -self.low / np.log(2)
        X, X2 = rest * p * x, rest * p * x * x
        self.eS = 2.0 ** -22 + 2.1 * U * X + ADD
        self.eH = self.eS + np.log(2) * (X * (2.0 ** -22 + ADD + self.eS) + 2.1 * U * X2) + 6 * U * (self.lnS + X)
        self.p, self.ep = p, 2.0 ** -22 + 2.1 * U * x + self.eS + 4 * U

    def logp(self, y):
        """ln p of an entry at y, and its tolerance."""
        return y - self.lnS, self.eS + 4 * U * (1 + abs(y) + self.lnS)


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("low", [-2.3, -1.1, -1.7, -9.0])
def test_statistics(ctx, dt, low):
    """One row, by a cluster, and as many as are taken by a CTA each (one row that all share)."""
    torch = need_gpu()
    r = Row(dt, low)
    for n in (1, 40, 320):
        tok = torch.tensor([0, V - 1], dtype=torch.int32, device="cuda").repeat(n)[:n].contiguous()
        lp, h = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        ctx.token_logprob(r.z.expand(n, V), tok, lp, h)
        ctx.sync()
        for first, y in ((0, 0.0), (1, r.low)):
            want, tol = r.logp(y)
            assert float((lp[first::2].double() - want).abs().max() if n > first else 0) <= tol
        assert float((h.double() - r.H).abs().max()) <= r.eH


def test_gradient(ctx):
    """Both sweeps: rows that a cluster takes one after another, and one row alone."""
    torch = need_gpu()
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    r = Row("bf16", -2.3)
    want, tol = r.logp(0.0)
    at_low = r.z[0] != 0
    for n in (160, 1):
        tok = torch.zeros(n, dtype=torch.int32, device="cuda")
        logp, stats, one = torch.empty(n, device="cuda"), torch.empty(5, device="cuda"), torch.ones(n, device="cuda")
        g = torch.empty((n, V), dtype=torch.bfloat16, device="cuda")
        ctx.learn_token_ppo(r.z.expand(n, V), tok, one * want, one, g, stats, weight=one, logp_out=logp,
                            grad_scale=2.0 ** 24)
        ctx.sync()
        assert float((logp.double() - want).abs().max()) <= tol
        e_rho = tol + U * abs(want) + 4 * U                       # ln p, the old one's rounding, exp
        assert abs(float(stats[1]) / n + 1) <= e_rho + 4 * U
        p = r.p * 2.0 ** 24                                       # slope -1: p of every entry but the token
        for i in {0, n // 2, n - 1}:
            low = g[i][at_low]
            assert bool((low == low[0]).all())
            assert abs(float(low[0]) - p) <= p * (2.0 ** -8 + r.ep + e_rho + 8 * U)
