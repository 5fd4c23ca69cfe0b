"""The token losses over no rows: valid for every vocabulary and type, with statistics of 0."""
import numpy as np
import pytest

from gpu_util import context, need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [1, 8, 100, 5000, 6145, 12_289, 32_768, 151_111, 1 << 24])
def test_no_rows_of_any_length(V, dt):
    torch = need_gpu()
    z = torch.empty((0, V), device="cuda", dtype=getattr(torch, dt))
    none = torch.empty(0, device="cuda")
    tok = none.int()
    with context() as ctx:
        for g in (z, None):
            s = [torch.full((k,), 9.0, device="cuda") for k in (5, 3, 3, 5)]
            ctx.token_logprob(z, tok, none, none)
            ctx.learn_token_ppo(z, tok, none, none, g, s[0], weight=none, ref_logp=none)
            for stats, top in ((s[1], 4), (s[2], 1024)):
                ids = torch.empty((0, top), dtype=torch.int32, device="cuda")
                ctx.learn_token_distill(z, ids, torch.empty((0, top), device="cuda"), g, stats)
            ctx.learn_token_pref(z, tok, torch.zeros(5, dtype=torch.int64, device="cuda"), g, s[3])
            ctx.learn_token_ppo(z, tok, none, none, g, None)                 # nothing to write at all
            ctx.sync()
            assert not s[0].any() and not s[1].any() and not s[2].any()
            np.testing.assert_allclose(s[3].tolist(), [2, np.log(2), 0, 0, 0], rtol=1e-6)
