"""Keys and values that are not finite in draft trees: what the nodes that see them give, and the others."""
import numpy as np
import pytest

import window_calls as calls
import window_dense as dense
from serving_inputs import PS, typed
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("where", ["window", "node", "path", "node, no window"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_positions_that_a_node_does_not_see(ada, dtype, where, bad):  # noqa: F811
    """One position's key and value (in bf16 its key alone) are not finite: nodes off its path, and those whose window it
    has left, are as without it; those that see a NaN are NaN."""
    rng = np.random.default_rng([len(where), 3])
    d, hq, hkv, new, ctx, sinks = 128, 4, 2, [100, 60], [300, 40], 4
    window = {"path": 9, "node, no window": 2 ** 31 - 1}.get(where, 100)
    cache, trees, q = calls.case(rng, "tree", dtype, d, hq, hkv, new, ctx, window, sinks)
    if where.startswith("node"):
        r, at = 0, ctx[0] + 11
        slot = (11,)
        pools = (trees.k, trees.v)
    else:
        # a place of the prefix that the root sees and deep nodes have left, or a node that those far behind it on its path have
        r, at = (0, ctx[0] - window + 4) if where == "window" else (1, ctx[1] + 2)
        slot = (cache.table[r, at // PS], slice(None), at % PS) if where == "window" else (new[0] + 2,)
        pools = (cache.k, cache.v) if where == "window" else (trees.k, trees.v)
    clean = dense.expected("tree", cache, trees, q, new, ctx, 0.09, window, sinks)
    value = typed(np.full(1, bad, np.float32), dtype)[0]
    for pool in pools if dtype == "f32" else pools[:1]:
        pool[slot] = value
    a = int(trees.indptr[r])
    seen = dense.seen_positions("tree", new[r], ctx[r], window, sinks, trees.parent[a:a + new[r]])[:, at]
    without = np.ones(sum(new), bool)
    without[a:a + new[r]] = ~seen
    assert seen.any() and (~seen).sum() > 10
    got = calls.run(ada, "tree", dtype, cache, trees, q, new, ctx, 0.09, window, sinks)
    calls.check("tree", dtype, got[without], tuple(x[without] for x in clean), 500)
    if np.isnan(bad):
        assert np.isnan(got[~without]).all()
