"""Attention over a window and sinks against fp64: prompts, single tokens and
draft trees, where windows, sinks, pages, tiles and requests begin and end."""
import numpy as np
import pytest

import window_calls as calls
from paged_calls import starts
from serving_inputs import PS, Cache, back, to_dev, typed
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

KINDS = ["prompt", "decode", "tree"]
DTYPES = ["bf16", "f32"]
# new rows (nodes), cached positions: before the nodes, the rows' own among them otherwise
NEW = [1, 7, 40, 70]
CTX = [1, 90, 333, 700]


def _lens(kind):
    return (NEW, [max(c, n) if kind == "prompt" else c for n, c in zip(NEW, CTX)])


@pytest.mark.parametrize("sinks", [0, 1, 4, 16, 17, 70, 2 ** 31 - 1])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 31, 33, 64, 100, 255, 2 ** 31 - 1])
@pytest.mark.parametrize("kind", KINDS)
def test_means(ada, kind, window, sinks):  # noqa: F811
    """The mean of what is seen: a position too many or too few shows."""
    new, ctx = _lens(kind)
    for i, dtype in enumerate(DTYPES):
        rng = np.random.default_rng([window, sinks, i])
        d, hq, hkv = [(128, 8, 2), (64, 4, 4)][(window + sinks + i) % 2]
        cache, trees, q = calls.case(rng, kind, dtype, d, hq, hkv, new, ctx, window, sinks, whole=True)
        got = calls.run(ada, kind, dtype, cache, trees, q, new, ctx, 0.1, window, sinks)
        out, size, _ = calls.expected(kind, cache, trees, q, new, ctx, 0.1, window, sinks)
        over = float((np.abs(got - out) - calls.mean_bound(kind, dtype, out, size)).max())
        assert over <= 0, over


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,hq,hkv", [(128, 32, 8), (128, 7, 1), (64, 16, 16), (64, 10, 2), (128, 16, 1), (64, 28, 4)])
@pytest.mark.parametrize("kind", KINDS)
def test_heads(ada, kind, d, hq, hkv, dtype):  # noqa: F811
    rng = np.random.default_rng([d, hq, hkv])
    new, ctx, window, sinks = [5, 33], [200, 50], 60, 3
    cache, trees, q = calls.case(rng, kind, dtype, d, hq, hkv, new, ctx, window, sinks)
    got = calls.run(ada, kind, dtype, cache, trees, q, new, ctx, d ** -0.5, window, sinks)
    calls.check(kind, dtype, got, calls.expected(kind, cache, trees, q, new, ctx, d ** -0.5, window, sinks), 800)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new,ctx,window,sinks", [
    ([300], [1500], 512, 4), ([1], [5000], 4096, 4), ([3], [4000], 100, 0), ([130, 1, 0, 64], [130, 900, 0, 2000], 257, 20),
    ([600], [600], 129, 1), ([17] * 9, [400 + 37 * i for i in range(9)], 300, 5), ([128], [2500], 2048, 130),
])
@pytest.mark.parametrize("kind", KINDS)
def test_lengths(ada, kind, new, ctx, window, sinks, dtype):  # noqa: F811
    rng = np.random.default_rng([len(new), window])
    if kind == "tree":
        new = [min(max(n, 1), 128) for n in new]
    d, hq, hkv = 128, 4, 2
    cache, trees, q = calls.case(rng, kind, dtype, d, hq, hkv, new, ctx, window, sinks)
    got = calls.run(ada, kind, dtype, cache, trees, q, new, ctx, d ** -0.5, window, sinks)
    calls.check(kind, dtype, got, calls.expected(kind, cache, trees, q, new, ctx, d ** -0.5, window, sinks), 6000)


@pytest.mark.parametrize("seed", range(24))
@pytest.mark.parametrize("kind", KINDS)
def test_drawn(ada, kind, seed):  # noqa: F811
    rng = np.random.default_rng([seed, KINDS.index(kind)])
    B = int(rng.integers(1, 7))
    new = [int(x) for x in rng.integers(1 if kind == "tree" else 0, 120, B)]
    if sum(new) == 0:
        new[0] = 1
    ctx = [int(x) + (n if kind == "prompt" else 0) for x, n in zip(rng.integers(0, 900, B), new)]
    window, sinks = int(np.exp(rng.uniform(0, 6.5))), int(rng.choice([0, 1, 4, 20, 64]))
    d, dtype = int(rng.choice([64, 128])), str(rng.choice(DTYPES))
    hkv = int(rng.choice([1, 2, 3]))
    hq = hkv * int(rng.choice([1, 2, 4, 5]))
    cache, trees, q = calls.case(rng, kind, dtype, d, hq, hkv, new, ctx, window, sinks)
    got = calls.run(ada, kind, dtype, cache, trees, q, new, ctx, d ** -0.5, window, sinks)
    calls.check(kind, dtype, got, calls.expected(kind, cache, trees, q, new, ctx, d ** -0.5, window, sinks), 1100)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind,many", [("prompt", 140), ("decode", 1100), ("tree", 170)])
def test_many_requests(ada, kind, many, dtype):  # noqa: F811
    """More requests than the tables and schedules of the other calls hold."""
    rng = np.random.default_rng(many)
    new = [int(x) for x in rng.integers(1, 4, many)]
    ctx = [int(x) + 3 for x in rng.integers(0, 150, many)]
    if kind == "decode":
        ctx[5], ctx[-1] = 0, 0
    cache, trees, q = calls.case(rng, kind, dtype, 64, 2, 1, new, ctx, 40, 4)
    got = calls.run(ada, kind, dtype, cache, trees, q, new, ctx, 0.125, 40, 4)
    calls.check(kind, dtype, got, calls.expected(kind, cache, trees, q, new, ctx, 0.125, 40, 4), 200)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", KINDS)
def test_a_window_over_everything_is_the_call_without_one(ada, kind, dtype):  # noqa: F811
    import torch
    rng = np.random.default_rng(3)
    new, ctx = _lens(kind)
    cache = Cache(rng, ctx, 2, 128, dtype)
    trees = calls.Trees(rng, new, 2, 128, dtype)
    q = typed(rng.standard_normal((4 if kind == "decode" else sum(new), 8, 128)), dtype)
    got = calls.run(ada, kind, dtype, cache, trees, q, new, ctx, 0.09, 770, 0)
    dev = dict(k_pages=to_dev(cache.k), v_pages=to_dev(cache.v), block_table=to_dev(cache.table), sm_scale=0.09, q=to_dev(q))
    dev["out"] = torch.empty_like(dev["q"])
    ctx32, code = np.asarray(ctx, np.int32), calls.code(ada, dtype)
    if kind == "prompt":
        ws = calls.workspace(ada.adaserve_prompt_attn_workspace_bytes(starts(new), ctx32, 8, 2, 128, PS, code))
        ada.adaserve_prompt_attn(token_indptr=to_dev(starts(new)), token_indptr_host=starts(new), context_len=to_dev(ctx32),
                                 context_len_host=ctx32, workspace=ws, **dev)
    elif kind == "decode":
        ws = calls.workspace(ada.adaserve_decode_attn_workspace_bytes(4, 700, 8, 2, 128, PS, code))
        ada.adaserve_decode_attn(context_len=to_dev(ctx32), max_context=700, workspace=ws, **dev)
    else:
        ws = calls.workspace(ada.adaserve_tree_attn_workspace_bytes(starts(new), ctx32, 8, 2, 128, PS, code))
        ada.adaserve_tree_attn_verify(node_indptr=to_dev(trees.indptr), node_indptr_host=trees.indptr, parent=to_dev(trees.parent),
                                      k_tree=to_dev(trees.k), v_tree=to_dev(trees.v), prefix_len=to_dev(ctx32),
                                      prefix_len_host=ctx32, workspace=ws, **dev)
    torch.cuda.synchronize()
    same = np.array_equal(got, calls.widen(back(dev["out"])))
    assert same


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("chunk", [False, True])
def test_prompt_positions_that_a_row_does_not_see(ada, bad, dtype, chunk):  # noqa: F811
    """One position's key and value are not finite: rows before it, and rows whose window it has left, are as without it."""
    rng = np.random.default_rng(17)
    n, c, window, sinks = (90, 600, 70, 4) if chunk else (500, 500, 150, 4)
    cache, _, q = calls.case(rng, "prompt", dtype, 128, 4, 2, [n], [c], window, sinks)
    at = c - n // 2
    page, slot = cache.table[0, at // PS], at % PS
    clean = calls.expected("prompt", cache, None, q, [n], [c], 0.09, window, sinks)
    value = typed(np.full(1, bad, np.float32), dtype)[0]
    cache.v[page, :, slot] = value
    cache.k[page, :, slot] = value
    got = calls.run(ada, "prompt", dtype, cache, None, q, [n], [c], 0.09, window, sinks)
    pos = c - n + np.arange(n)
    without = (at > pos) | ((at <= pos - window) & (at >= sinks))
    assert without.sum() > n // 4 and (~without).any()
    calls.check("prompt", dtype, got[without], tuple(x[without] for x in clean), 700)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", KINDS)
def test_pages_outside_the_pool_are_zeros(ada, kind, dtype):  # noqa: F811
    rng = np.random.default_rng(5)
    new, ctx, window, sinks = [3, 20], [300, 170], 90, 20
    cache, trees, q = calls.case(rng, kind, dtype, 64, 4, 2, new, ctx, window, sinks)
    cache.table[0, 0], cache.table[0, 17], cache.table[1, 9] = -1, cache.pages, -7
    got = calls.run(ada, kind, dtype, cache, trees, q, new, ctx, 0.125, window, sinks)
    calls.check(kind, dtype, got, calls.expected(kind, cache, trees, q, new, ctx, 0.125, window, sinks), 400)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sinks", [0, 2])
def test_rows_that_see_nothing(ada, dtype, sinks):  # noqa: F811
    rng = np.random.default_rng(6)
    cache, _, q = calls.case(rng, "prompt", dtype, 64, 4, 2, [20, 5], [7, 0], 3, sinks)
    got = calls.run(ada, "prompt", dtype, cache, None, q, [20, 5], [7, 0], 0.125, 3, sinks, pad=4)
    nothing = bool((got[:13] == 0).all() and (got[20:] == 0).all())
    assert nothing and bool((got[13:20] != 0).any(2).all())
    calls.check("prompt", dtype, got, calls.expected("prompt", cache, None, q, [20, 5], [7, 0], 0.125, 3, sinks), 20)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B", [4, 1100])
def test_decode_lengths_of_zero_and_outside_the_bound(ada, dtype, B):  # noqa: F811
    rng = np.random.default_rng(7)
    ctx = [40 + i % 60 for i in range(B)]
    ctx[1] = 0
    cache, _, q = calls.case(rng, "decode", dtype, 64, 4, 2, None, ctx, 30, 2)
    wrong = list(ctx)
    wrong[2], wrong[3] = 201, -1
    got = calls.run_decode(ada, q, wrong, cache, dtype, 0.125, 30, 2, most=200, table=np.pad(cache.table, ((0, 0), (0, 20)), constant_values=-1))
    out, size, reach = calls.expected("decode", cache, None, q, None, ctx, 0.125, 30, 2)
    assert bool((got[1] == 0).all()) and bool(np.isnan(got[2:4]).all())
    rest = [0] + list(range(4, B))
    calls.check("decode", dtype, got[rest], (out[rest], size[rest], reach[rest]), 120)


@pytest.mark.parametrize("new,ctx,window,sinks", [([200], [900], 300, 4), ([64], [3000], 2000, 0), ([700, 300], [700, 300], 200, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_scores_that_rise(ada, d, new, ctx, window, sinks):  # noqa: F811
    """Scores that grow along the keys, beyond what weights against a row's first keys can hold."""
    rng = np.random.default_rng(d)
    cache, _, _ = calls.case(rng, "prompt", "bf16", d, 4, 2, new, ctx, window, sinks)
    q = typed(rng.standard_normal((sum(new), 4, d)) * 0.05 + 1, "bf16")
    k = calls.widen(cache.k)
    for r, c in enumerate(ctx):
        for t in range(c):
            p = cache.table[r, t // PS]
            if 0 <= p < cache.pages and np.isfinite(k[p, :, t % PS]).all():
                k[p, :, t % PS] = (t / c) * 3 + rng.standard_normal((2, d)) * 0.01
    cache.k = typed(k.astype(np.float32), "bf16")
    got = calls.run(ada, "prompt", "bf16", cache, None, q, new, ctx, 1.0, window, sinks)
    calls.check("prompt", "bf16", got, calls.expected("prompt", cache, None, q, new, ctx, 1.0, window, sinks), 3000)


@pytest.mark.parametrize("scale", [-0.2, 0.0, 3e-7])
@pytest.mark.parametrize("kind", KINDS)
def test_f32_scales(ada, kind, scale):  # noqa: F811
    rng = np.random.default_rng(12)
    new, ctx, window, sinks = [9, 40], [300, 65], 50, 4
    cache, trees, q = calls.case(rng, kind, "f32", 64, 4, 2, new, ctx, window, sinks)
    got = calls.run(ada, kind, "f32", cache, trees, q, new, ctx, scale, window, sinks)
    calls.check(kind, "f32", got, calls.expected(kind, cache, trees, q, new, ctx, scale, window, sinks), 400)


@pytest.mark.parametrize("dtype", DTYPES)
def test_trees_longer_than_their_window(ada, dtype):  # noqa: F811
    """Chains, whose first nodes leave the window of the last ones, over short prefixes; some of them are sinks."""
    rng = np.random.default_rng(8)
    new, ctx = [128, 60, 1, 100], [3, 0, 0, 40]
    for window, sinks in [(1, 0), (20, 0), (33, 10), (5, 200)]:
        cache = Cache(rng, ctx, 2, 64, dtype)
        trees = calls.Trees(rng, new, 2, 64, dtype, chain=True)
        q = typed(rng.standard_normal((sum(new), 6, 64)), dtype)
        got = calls.run(ada, "tree", dtype, cache, trees, q, new, ctx, 0.125, window, sinks)
        calls.check("tree", dtype, got, calls.expected("tree", cache, trees, q, new, ctx, 0.125, window, sinks), 200)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["prompt", "decode"])
def test_rows_apart_on_another_stream(ada, kind, dtype):  # noqa: F811
    """Queries that are slices of a wider projection's rows, on a stream of their own."""
    import torch
    rng = np.random.default_rng(9)
    new, ctx, window, sinks = [3, 50], [80, 260], 100, 4
    cache, _, q = calls.case(rng, kind, dtype, 128, 4, 2, new, ctx, window, sinks)
    T = q.shape[0]
    wide = torch.full((T, 7, 128), float("nan"), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    wide[:, 1:5] = to_dev(q)
    out = torch.empty(T, 4, 128, dtype=wide.dtype, device="cuda")
    ctx32, indptr, code = np.asarray(ctx, np.int32), starts(new), calls.code(ada, dtype)
    dev = dict(k_pages=to_dev(cache.k), v_pages=to_dev(cache.v), block_table=to_dev(cache.table), context_len=to_dev(ctx32),
               window=window, sinks=sinks, sm_scale=0.09, q=wide[:, 1:5], out=out)
    indptr_dev = to_dev(indptr)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    if kind == "prompt":
        ws = calls.workspace(ada.adaserve_window_prompt_attn_workspace_bytes(indptr, ctx32, 4, 2, 128, PS, window, sinks, code))
        torch.cuda.synchronize()
        ada.adaserve_window_prompt_attn(token_indptr=indptr_dev, token_indptr_host=indptr, context_len_host=ctx32, workspace=ws,
                                        stream=stream, **dev)
    else:
        ws = calls.workspace(ada.adaserve_window_decode_attn_workspace_bytes(2, 260, 4, 2, 128, PS, window, sinks, code))
        torch.cuda.synchronize()
        ada.adaserve_window_decode_attn(max_context=260, workspace=ws, stream=stream, **dev)
    stream.synchronize()
    calls.check(kind, dtype, calls.widen(back(out)), calls.expected(kind, cache, None, q, new, ctx, 0.09, window, sinks), 400)


@pytest.mark.parametrize("dtype", DTYPES)
def test_decode_replayed_with_growing_lengths(ada, dtype):  # noqa: F811
    import torch
    rng = np.random.default_rng(10)
    B, hq, hkv, d, window, sinks, most = 5, 8, 2, 128, 100, 4, 700
    cache = Cache(rng, [most] * B, hkv, d, dtype)
    q = typed(rng.standard_normal((B, hq, d)), dtype)
    code = calls.code(ada, dtype)
    ws = calls.workspace(ada.adaserve_window_decode_attn_workspace_bytes(B, most, hq, hkv, d, PS, window, sinks, code))
    qd, lens = to_dev(q), to_dev(np.zeros(B, np.int32))
    out = torch.empty_like(qd)
    args = dict(q=qd, k_pages=to_dev(cache.k), v_pages=to_dev(cache.v), block_table=to_dev(cache.table), context_len=lens,
                max_context=most, window=window, sinks=sinks, sm_scale=0.09, out=out, workspace=ws)
    ada.adaserve_window_decode_attn(**args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ada.adaserve_window_decode_attn(**args)
    for step in range(5):
        ctx = [int(x) for x in rng.integers(0, most + 1, B)]
        lens.copy_(to_dev(np.asarray(ctx, np.int32)))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = calls.widen(back(out))
        calls.check("decode", dtype, got, calls.expected("decode", cache, None, q, None, ctx, 0.09, window, sinks), 700)
        ada.adaserve_window_decode_attn(**args)
        torch.cuda.synchronize()
        assert np.array_equal(got, calls.widen(back(out)))
