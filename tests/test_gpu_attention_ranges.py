"""Prompt and single-token attention at the ends of what their values and scales
may be."""
import numpy as np
import pytest

from paged_calls import check, run_decode, run_prompt, starts
from serving_inputs import Cache, typed
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def rising(rng, new, ctx, hq, hkv, d, dtype, nats, size, positive):
    """Scores around -nats / 2 for the first 40 keys and around nats / 2 after them; values of magnitude `size`."""
    c = Cache(rng, ctx, hkv, d, dtype)
    k = np.asarray(rng.standard_normal(c.k.shape) * 0.1, np.float32)
    v = np.asarray(rng.standard_normal(c.v.shape), np.float32)
    side = np.where(np.arange(c.table.shape[1] * 16) < 40, -1.0, 1.0).reshape(-1, 16)
    for row in c.table:
        for e, p in enumerate(row):
            if p >= 0:
                k[p, :, :, 0] = side[e] * 4
    c.k, c.v = typed(k, dtype), typed((np.abs(v) if positive else v) * size, dtype)
    q = rng.standard_normal((int(starts(new)[-1]), hq, d)) * 0.1
    q[:, :, 0] = nats / 2 / 4 * d ** 0.5
    return c, typed(q, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("positive", [True, False])
@pytest.mark.parametrize("new,ctx,split,d", [([200], [260], False, 128), ([120], [4000], True, 128), ([70, 40], [90, 1500], None, 64)])
def test_prompt_large_values_under_rising_scores(ada, dtype, positive, new, ctx, split, d):  # noqa: F811
    """Weights up to 2^52 of the first keys' times values of 2^70, some hundred of them, are beyond fp32; their
    quotient is not, and the sums of weights alone do not show it (2^61)."""
    rng = np.random.default_rng(sum(ctx) + positive)
    c, q = rising(rng, new, ctx, 8, 2, d, dtype, 36.0, 2.0 ** 70, positive)
    got = run_prompt(ada, q, new, ctx, c, dtype, d ** -0.5, split=split if dtype == "bf16" else False)
    check("prompt", got, q, new, ctx, c, dtype, d ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_large_values_under_rising_scores(ada, dtype):  # noqa: F811
    rng = np.random.default_rng(5)
    ctx = [260, 4000, 41]
    c, q = rising(rng, [1] * 3, ctx, 8, 2, 128, dtype, 36.0, 2.0 ** 70, True)
    got = run_decode(ada, q, ctx, c, dtype, 128 ** -0.5)
    check("decode", got, q, [1] * 3, ctx, c, dtype, 128 ** -0.5)


@pytest.mark.parametrize("new,ctx,split", [([200], [260], False), ([120], [4000], True)])
def test_prompt_values_at_the_documented_size(ada, new, ctx, split):  # noqa: F811
    """|value| * context just below 2^118."""
    rng = np.random.default_rng(11)
    c, q = rising(rng, new, ctx, 8, 2, 128, "bf16", 36.0, 1.0, True)
    c.v = typed(np.full(c.v.shape, 2.0 ** 118 / (ctx[0] + 1), np.float32), "bf16")
    got = run_prompt(ada, q, new, ctx, c, "bf16", 128 ** -0.5, split=split)
    check("prompt", got, q, new, ctx, c, "bf16", 128 ** -0.5)


@pytest.mark.parametrize("new,ctx,split", [([200], [260], False), ([120], [4000], True)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_far_scores_at_a_small_scale(ada, dtype, new, ctx, split):  # noqa: F811
    """Queries and keys of 2^47 at a scale of 2^-90: every score is about -3100, and they differ by units."""
    rng = np.random.default_rng(3)
    d, scale = 128, 2.0 ** -90
    c = Cache(rng, ctx, 2, d, dtype)
    c.k = typed(-2.0 ** 47 * (1 + 2.0 ** -7 * rng.integers(0, 3, c.k.shape)), dtype)
    q = typed(np.full((int(starts(new)[-1]), 8, d), 1.5 * 2.0 ** 47), dtype)
    got = run_prompt(ada, q, new, ctx, c, dtype, scale, split=split if dtype == "bf16" else False)
    check("prompt", got, q, new, ctx, c, dtype, scale)
