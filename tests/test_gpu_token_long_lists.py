"""Distillation with long lists over more rows than the device holds at once, and preference calls
of few pairs with many rows of a long vocabulary, against the 64-bit oracle."""
import pytest

from gpu_util import context
from test_gpu_token_losses import Batch, Distill, Pref, check_distill, check_pref, empty

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = context()
    yield c
    c.sync()
    c.close()


@pytest.mark.parametrize("n,V,dt,top", [(700, 32_768, "bf16", 1024), (500, 20_003, "f32", 450), (330, 60_001, "f16", 600),
                                        (320, 100_000, "bf16", 500), (170, 50_001, "f32", 1024)])
def test_long_lists_over_many_rows(ctx, n, V, dt, top):
    b = Batch(n, V, dt, n + top, T=1.2, out=0.0)
    check_distill(ctx, b, top, tdt=dt)
    d, first = Distill(b, top, twice=True), None
    for _ in range(2):
        (_, g), stats = b.grad(pad=1), empty(3)
        d.call(ctx, b, g, stats=stats)
        ctx.sync()
        first = first or (g, stats)
        assert bool((g == first[0]).all()) and bool((stats == first[1]).all())


@pytest.mark.parametrize("n,V,dt,pairs", [(2000, 20_000, "bf16", 1), (1500, 20_001, "f32", 2), (20_000, 700, "f16", 3),
                                          (50_000, 40, "f32", 1)])
def test_few_pairs_of_many_rows(ctx, n, V, dt, pairs):
    b = Batch(n, V, dt, n + V, T=0.9, masked=0.1, out=0.3)
    check_pref(ctx, b, pairs, beta=0.01)
    p, first = Pref(b, pairs), None
    for _ in range(2):
        (_, g), stats, reward = b.grad(), empty(5), empty(2 * pairs)
        p.call(ctx, b, g, reward=reward, stats=stats)
        ctx.sync()
        first = first or (g, stats, reward)
        assert all(bool((x == y).all()) for x, y in zip((g, stats, reward), first))
