"""The bounds that attention on the GPU is held to, against planted mistakes (in the oracle, on the CPU)."""
import numpy as np
import pytest

from marked_caches import counted, mean_bound, means, pointed
from oracle import serving
from paged_calls import bound, reach, starts
from serving_inputs import PS, Cache, bf16_bits, typed

MISTAKES = ["wrong page", "a key too few", "the last block missing", "a page twice"]


def mistaken(which, table, ctx):
    """The table and length that a wrong kernel would have read."""
    t, c = table.copy(), list(ctx)
    pages = -(-c[0] // PS)
    if which == "wrong page":
        t[0, pages // 2] = t[0, 3]
    elif which == "a key too few":
        c[0] -= 1
    elif which == "the last block missing":
        c[0] -= 32
    else:
        t[0, pages - 2] = t[0, pages - 3]
    return t, c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [129, 4097, 9000, 20000])
@pytest.mark.parametrize("which", MISTAKES)
def test_mistakes_show_in_means(dtype, length, which):
    rng = np.random.default_rng(length)
    c = counted(rng, [length], 2, 128, dtype)
    right = means(c, [1], [length], 8)
    table, ctx = mistaken(which, c.table, [length])
    wrong = means(c, [1], ctx, 8, table)
    assert (np.abs(wrong - right) > 2 * mean_bound(dtype, right)).mean() > 0.1   # at many columns, at twice the bound
    sums = right * length
    assert np.abs(sums - np.rint(sums)).max() < 1e-6 and np.abs(sums).max() < 2 ** 24


@pytest.mark.parametrize("kind", ["prompt", "decode"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [129, 4097, 20000])
@pytest.mark.parametrize("which", MISTAKES[1:3])
def test_mistakes_show_in_pointed_queries(kind, dtype, length, which):
    rng = np.random.default_rng(length)
    d, scale = 128, 128 ** -0.5
    c, q = pointed(rng, [1], [length], 8, 2, d, dtype)
    out, size, _ = serving.paged_attention(q, [0, 1], c.k, c.v, c.table, [length], scale)
    b = bound(kind, dtype, out, size, reach(q, [0, 1], c, c.table, [length], scale), length, d)
    table, ctx = mistaken(which, c.table, [length])
    wrong, _, _ = serving.paged_attention(q, [0, 1], c.k, c.v, table, ctx, scale)
    assert (np.abs(wrong - out) > 4 * b)[:, 0].mean() > 0.5       # head 0 looks at the last key


@pytest.mark.parametrize("ctx", [[17, 40, 3], [129, 300]])
def test_weights_in_one_bf16_part_show(ctx):
    """Single tokens hold their weights in two bf16 parts: with the first alone they are beyond their bound."""
    rng = np.random.default_rng(sum(ctx))
    d, scale = 128, 128 ** -0.5
    c = Cache(rng, ctx, 2, d, "bf16")
    q = typed(rng.standard_normal((len(ctx), 8, d)), "bf16")
    indptr = starts([1] * len(ctx))
    out, size, _ = serving.paged_attention(q, indptr, c.k, c.v, c.table, ctx, scale)
    most = reach(q, indptr, c, c.table, ctx, scale)
    wide, k, v = (serving.widen(x) for x in (q, c.k, c.v))
    wrong = np.zeros_like(out)
    for r, n in enumerate(ctx):
        at = np.arange(n)
        for h in range(8):
            z = wide[r, h] @ k[c.table[r][at // PS], h // 4, at % PS].T * scale
            w = np.exp(z - z.max())
            part = serving.widen(bf16_bits(w))
            wrong[r, h] = part @ v[c.table[r][at // PS], h // 4, at % PS] / w.sum()
    assert (np.abs(wrong - out) > bound("decode", "bf16", out, size, most, max(ctx), d)).any()
    assert (np.abs(wrong - out) <= bound("prompt", "bf16", out, size, most, max(ctx), d)).all()   # what prompts do
