"""More rows, and more pairs, than an ordinary call has: sums of millions of terms, counts past 31 bits."""
import numpy as np
import pytest

from gpu_util import context, need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_ref", [False, True])
def test_reward_of_very_many_rows(with_ref):
    """An answer of 2^28 rows, 2 million for a thread, over one row of logits that all share."""
    torch = need_gpu()
    n = 1 << 28
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    z = torch.tensor([[0.25, 0.0]], device="cuda")
    tok = torch.zeros(n, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, n, n], device="cuda")
    ref = torch.full((n,), 0.3125, device="cuda") if with_ref else None
    reward, stats = torch.empty(2, device="cuda"), torch.empty(5, device="cuda")
    with context() as ctx:
        ctx.learn_token_pref(z.expand(n, 2), tok, off, None, stats, ref_logp=ref, reward_out=reward, beta=2.0 ** -20)
        ctx.sync()
    # ln p of 0.58 to 2^-22 + 2 u for S, 4 u (1 + 0.58 + 0.58) besides; the sum's rounding and beta's product
    lp = -np.log1p(np.exp(-0.25))
    want = (lp - (0.3125 if with_ref else 0)) * 2.0 ** 8
    tol = 2.0 ** 8 * (2.0 ** -22 + 11 * 2.0 ** -24) + 2 * 2.0 ** -24 * abs(want)
    assert abs(float(reward[0]) - want) <= tol and float(reward[1]) == 0
