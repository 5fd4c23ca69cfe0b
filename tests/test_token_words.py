"""Whole numbers of the token calls that do not fit their 32 bits: refused, not taken modulo 2^32."""
import pytest

from paper_2106_07551_gb300 import Context


class Fake:
    """A context whose library must not be called."""
    handle = None

    @property
    def lib(self):
        raise AssertionError("the call went through")


@pytest.mark.parametrize("more", [dict(agent=2 ** 32), dict(agent=2 ** 32 + 3), dict(top_k=2 ** 32), dict(top_k=2 ** 33 + 50),
                                  dict(agent=-2 ** 31 - 1)])
def test_draws(more):
    import torch
    z, out = torch.zeros((3, 8)), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="32 bits"):
        Context.token_sample(Fake(), z, out, uniform=torch.zeros(3), **more)
    with pytest.raises(AssertionError):                  # what fits is the library's to refuse
        Context.token_sample(Fake(), z, out, uniform=torch.zeros(3), agent=2 ** 31, top_k=-1)


@pytest.mark.parametrize("site", [2 ** 32, 2 ** 40 + 1, -2 ** 31 - 1])
def test_dropout(site):
    import torch
    x, seq, step = torch.zeros((3, 8)), torch.zeros(3, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="32 bits"):
        Context.dropout(Fake(), x, torch.empty_like(x), 0.1, 1, site=site, sequence=seq, step=step)
    with pytest.raises(AssertionError):
        Context.dropout(Fake(), x, torch.empty_like(x), 0.1, 1, site=2 ** 15, sequence=seq, step=step)
