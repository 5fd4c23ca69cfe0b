"""The example's rollout, dropout and gradient of a loss of its own."""
import importlib.util
import pathlib

import numpy as np
import pytest

from gpu_util import context
from oracle import token_rollout as tr

pytestmark = pytest.mark.gpu
PATH = pathlib.Path(__file__).resolve().parents[1] / "examples" / "token_policy.py"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("token_policy_steps", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_answers_do_not_hang_on_their_batch(example):
    """The same numbers, prompts and weights give the same answers, alone or among others; every answer ends
    at its own length."""
    import torch
    ctx, n = context(), 20
    policy = example.Policy(500, 1)
    prompts = torch.arange(n, device="cuda") % example.PROMPTS
    made = []
    for count in (n, n, 7):
        gen = torch.Generator(device="cuda").manual_seed(3)
        example.Answers.made = 100
        made.append(example.Answers(ctx, policy, prompts[:count], gen, drop=True))
    ctx.sync()
    a, b, c = made
    assert bool((a.tokens == b.tokens).all()) and bool((a.logp == b.logp).all())
    assert bool(((a.tokens >= 0).view(n, -1).sum(1) == a.length).all())
    # another batch's network may round the logits apart; the masks are the same
    keep = tr.dropout_keep(example.HIDDEN, example.DROP, example.SEED, 0, a.number.cpu().numpy(),
                           a.position.cpu().numpy().astype(np.int32))
    ones = torch.ones((n * example.LENGTH, example.HIDDEN), device="cuda")
    out = example.Dropout.apply(ones, ctx, a.number, a.position.int())
    few = example.Dropout.apply(ones[:7 * example.LENGTH], ctx, c.number, c.position.int())
    ctx.sync()
    np.testing.assert_array_equal(out.cpu().numpy() > 0, keep)
    assert bool((few == out[:7 * example.LENGTH]).all())
    ctx.close()


def test_gradients(example):
    """Of dropout, and of a loss of ln p and H, against the same in 64-bit autograd."""
    import torch
    ctx, n, V = context(), 9, 40
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((n, example.HIDDEN), generator=gen, device="cuda", requires_grad=True)
    w = torch.randn((n, example.HIDDEN), generator=gen, device="cuda")
    seq, at = torch.arange(n, device="cuda"), torch.full((n,), 2, dtype=torch.int32, device="cuda")
    (example.Dropout.apply(x, ctx, seq, at) * w).sum().backward()
    ctx.sync()
    least = tr.dropout_least(example.DROP)
    keep = tr.dropout_keep(example.HIDDEN, example.DROP, example.SEED, 0, seq.cpu().numpy(), at.cpu().numpy())
    want = np.where(keep, w.double().cpu().numpy() * 65536 / (65536 - least), 0)
    assert (np.abs(x.grad.cpu().numpy() - want) <= 3 * U * np.abs(want)).all()   # the factor's and the product's rounding
    z = torch.randn((n, V), generator=gen, device="cuda", requires_grad=True)
    tokens = torch.randint(0, V, (n,), generator=gen, device="cuda", dtype=torch.int32)
    logp, entropy = example.Scores.apply(z, ctx, tokens)
    (0.1 * entropy - logp).sum().backward()
    ctx.sync()
    y = z.detach().double().requires_grad_(True)
    lp = torch.log_softmax(y, 1)
    (-0.1 * (lp.exp() * lp).sum(1) - lp.gather(1, tokens[:, None].long())[:, 0]).sum().backward()
    # |slopes| at most 1 and 0.1 (|ln p| + H) p; p is good to 2^-22 and some twenty roundings
    size = lp.exp() * (1 + 0.1 * (lp.abs() + 2 * np.log(V) + 1)) + 0.0
    size.scatter_add_(1, tokens[:, None].long(), torch.ones((n, 1), device="cuda", dtype=torch.float64))
    assert bool(((z.grad.double() - y.grad).abs() <= (2 ** -22 + 100 * U) * size).all())
    ctx.close()
