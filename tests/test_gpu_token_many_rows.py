"""More rows, and more pairs, than an ordinary call has: sums of millions of terms, counts past 31 bits."""
import ctypes as C

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


def test_as_many_pairs_as_are_taken():
    """2^30 pairs, whose last offset is entry 2^31: pairs without rows but the last, whose two answers
    have a row each."""
    torch = need_gpu()
    from paper_2106_07551_gb300 import _abi
    P = 1 << 30
    if torch.cuda.mem_get_info()[0] < 32 << 30:
        pytest.skip("needs 32 GB")
    off = torch.zeros(2 * P + 1, dtype=torch.int64, device="cuda")
    off[2 * P - 1], off[2 * P] = 1, 2
    z = torch.tensor([[1.0, 0.0], [0.0, 1.0]], device="cuda")
    tok, stats, reward = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.empty(5, device="cuda"), torch.empty(
        2 * P, device="cuda")
    g = torch.empty_like(z)
    with context() as ctx:
        ctx.learn_token_pref(z, tok, off, g, stats, reward_out=reward, beta=2.0, grad_scale=float(P))
        ctx.sync()
        s = stats.double().cpu().numpy()
        assert s[0] == P
        np.testing.assert_allclose(s[1], np.log(2), rtol=1e-6)
        # D = 2 (ln p(0 | 1, 0) - ln p(0 | 0, 1)) = 2: slope -2 s(-2), times 1 - p(0) in each row
        np.testing.assert_allclose(reward[-2:].tolist(), [-2 * np.log1p(np.exp(-1)), -2 * np.log1p(np.exp(1))], rtol=1e-5)
        assert not reward[:-2].any()
        want = -2 / (1 + np.exp(2)) * np.array([1 / (1 + np.e), -1 / (1 + np.exp(-1))])
        np.testing.assert_allclose(g[:, 0].tolist(), want, rtol=1e-5)
        np.testing.assert_allclose(g[:, 1].tolist(), -want, rtol=1e-5)
        b = _abi.TokenBatch(z.data_ptr(), tok.data_ptr(), 2, 2, 2, 0, 1.0)
        p = _abi.TokenPref(off.data_ptr(), None, P + 1, 1.0, 0.0)
        assert ctx.lib.malib_learn_token_pref(ctx.handle, C.byref(b), C.byref(p), None, None, None) == _abi.MALIB_EINVAL


def test_rows_past_31_bits_are_counted():
    """2^31 + 77 rows over one row of logits that all share."""
    torch = need_gpu()
    n = (1 << 31) + 77
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB")
    z = torch.zeros((1, 2), dtype=torch.bfloat16, device="cuda").expand(n, 2)
    tok = torch.zeros(n, dtype=torch.int32, device="cuda")
    tok[5] = -1
    old = torch.zeros(n, device="cuda")                           # and the advantages
    old[n - 1] = 1.0
    stats = torch.empty(5, device="cuda")
    with context() as ctx:
        ctx.learn_token_ppo(z, tok, old, old, None, stats)
        ctx.sync()
    s = stats.double().cpu().numpy()
    assert s[0] == np.float32(n - 1)
    # the last row: rho = e^-1 / 2, A = 1, weight 1 / n; every row's entropy is ln 2
    np.testing.assert_allclose(s[1], -0.5 * np.exp(-1) / n, rtol=1e-5)
    np.testing.assert_allclose(s[4], np.log(2), rtol=1e-6)


@pytest.mark.parametrize("n", [(1 << 40) + 1, 1 << 58, (1 << 59) + 3, 1 << 60, (1 << 60) + 1, (1 << 63) - 1])
def test_rows_that_no_memory_holds_are_refused(n):
    """Rows that share one row of logits have no extent that could overflow; their work space has."""
    torch = need_gpu()
    from paper_2106_07551_gb300 import _abi
    z, v = torch.zeros((1, 8), device="cuda"), torch.zeros(8, device="cuda")
    i, off = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    p, q, d = _abi.TokenPpo(v.data_ptr(), v.data_ptr(), None, None, 0.2, 0.2, 0.0, 0.0), _abi.TokenPref(
        off.data_ptr(), None, 1, 0.1, 0.0), _abi.TokenDistill(i.data_ptr(), v.data_ptr(), None, 1, 0)
    b = _abi.TokenBatch(z.data_ptr(), i.data_ptr(), n, 0, 8, 0, 1.0)
    t = _abi.TokenBatch(z.data_ptr(), None, n, 0, 8, 0, 1.0)
    with context() as ctx:
        lib, h, r = ctx.lib, ctx.handle, C.byref
        assert lib.malib_token_logprob(h, r(b), v.data_ptr(), None) == _abi.MALIB_EINVAL
        assert lib.malib_learn_token_ppo(h, r(b), r(p), None, None, v.data_ptr()) == _abi.MALIB_EINVAL
        assert lib.malib_learn_token_pref(h, r(b), r(q), None, None, v.data_ptr()) == _abi.MALIB_EINVAL
        assert lib.malib_learn_token_distill(h, r(t), r(d), None, None, v.data_ptr()) == _abi.MALIB_EINVAL
        assert "n_rows" in ctx.last_error()
        ctx.sync()
