"""What the attentions over a window are held to, against planted mistakes (in the references, on the CPU)."""
import numpy as np
import pytest

import window_calls as calls
import window_dense as dense
from oracle.serving import widen
from serving_inputs import typed

NEW, CTX, WINDOW, SINKS = [9, 20], [900, 2100], 1500, 4


@pytest.mark.parametrize("kind,new,ctx,window,sinks", [
    ("prompt", [5, 0, 40], [7, 3, 90], 11, 2), ("prompt", [9], [4], 3, 0), ("prompt", [30], [80], 500, 0),
    ("tree", [6, 30], [0, 75], 13, 4), ("tree", [20], [10], 1, 0),
])
def test_dense_references_are_the_oracles(kind, new, ctx, window, sinks):
    """Two references, written apart."""
    rng = np.random.default_rng([len(new), window])
    cache, trees, q = calls.case(rng, kind, "f32", 64, 4, 2, new, ctx, window, sinks)
    cache.table[0, 0] = -1
    for x, y in zip(dense.expected(kind, cache, trees, q, new, ctx, 0.1, window, sinks, "cpu"),
                    calls.expected(kind, cache, trees, q, new, ctx, 0.1, window, sinks)):
        assert np.abs(x - y).max() < 1e-12


def test_chunks_rounded_to_bf16_show():
    """Means of split prefixes whose chunks' outputs are rounded to bf16 are beyond their bound at many columns, those whose
    chunks' outputs are fp32 nowhere."""
    rng = np.random.default_rng(0)
    cache, trees, q = calls.case(rng, "tree", "bf16", 128, 2, 2, NEW, CTX, WINDOW, SINKS, whole=True)
    out, size, _ = dense.expected("tree", cache, trees, q, NEW, CTX, 0.09, WINDOW, SINKS, "cpu")
    v, vt = widen(cache.v), widen(trees.v)
    r, a, n, c = 1, NEW[0], NEW[1], CTX[1]
    at = np.arange(c)
    page = np.clip(cache.table[r][at // 16], 0, cache.pages - 1)
    seen = dense.seen_positions("tree", n, c, WINDOW, SINKS, trees.parent[a:])
    far = {}
    for rounding in ("bf16", "f32"):
        got = np.zeros_like(out[a:])
        for g in range(2):
            values = np.concatenate([v[page, g, at % 16], vt[a:, g]])
            for i in range(n):
                keys = np.flatnonzero(seen[i])
                parts = np.array_split(keys, 2)
                means = [widen(typed(values[p].mean(0).astype(np.float32), rounding)) for p in parts]
                got[i, g] = sum(len(p) * m for p, m in zip(parts, means)) / len(keys)
        far[rounding] = np.abs(got - out[a:]) > dense.split_mean_bound(out[a:], size[a:])
    assert far["bf16"].mean() > 0.1 and not far["f32"].any()
