"""Calls of the attentions over a window on given queries and caches, and how far
their results may be from fp64's."""
import numpy as np

from oracle import window as oracle
from oracle.serving import widen
from paged_calls import SENTINEL, starts
from serving_inputs import PS, Cache, back, to_dev, typed


def code(ada, dtype):
    return ada.ADASERVE_BF16 if dtype == "bf16" else ada.ADASERVE_F32


def workspace(need):
    import torch
    return torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None


def run_prompt(ada, q, new, ctx, cache, dtype, scale, window, sinks, table=None, pad=0):
    import torch
    T, hq, d = q.shape
    indptr, ctx32 = starts(new), np.asarray(ctx, np.int32)
    table = cache.table if table is None else table
    need = ada.adaserve_window_prompt_attn_workspace_bytes(indptr, ctx32, hq, cache.k.shape[1], d, PS, window, sinks, code(ada, dtype))
    rows = to_dev(np.concatenate([q, np.zeros((pad, hq, d), q.dtype)]))
    out = torch.full(rows.shape, SENTINEL, dtype=rows.dtype, device="cuda")
    print("window prompt rows", T, "of", len(ctx32), "heads", hq, cache.k.shape[1], "D", d, dtype, "window", window, sinks,
          "workspace", need, flush=True)
    ada.adaserve_window_prompt_attn(token_indptr=to_dev(indptr), token_indptr_host=indptr, q=rows, k_pages=to_dev(cache.k),
                                    v_pages=to_dev(cache.v), block_table=to_dev(table), context_len=to_dev(ctx32),
                                    context_len_host=ctx32, window=window, sinks=sinks, sm_scale=scale, out=out,
                                    workspace=workspace(need))
    torch.cuda.synchronize()
    got = widen(back(out))
    assert (got[T:] == SENTINEL).all()
    return got[:T]


def run_decode(ada, q, ctx, cache, dtype, scale, window, sinks, table=None, most=None):
    import torch
    B, hq, d = q.shape
    ctx32 = np.asarray(ctx, np.int32)
    table = cache.table if table is None else table
    most = int(ctx32.max(initial=0)) if most is None else most
    need = ada.adaserve_window_decode_attn_workspace_bytes(B, most, hq, cache.k.shape[1], d, PS, window, sinks, code(ada, dtype))
    rows = to_dev(q)
    out = torch.full(rows.shape, SENTINEL, dtype=rows.dtype, device="cuda")
    print("window decode requests", B, "heads", hq, cache.k.shape[1], "D", d, dtype, "window", window, sinks, "workspace", need,
          flush=True)
    ada.adaserve_window_decode_attn(q=rows, k_pages=to_dev(cache.k), v_pages=to_dev(cache.v), block_table=to_dev(table),
                                    context_len=to_dev(ctx32), max_context=most, window=window, sinks=sinks, sm_scale=scale,
                                    out=out, workspace=workspace(need))
    torch.cuda.synchronize()
    return widen(back(out))


class Trees:
    """Draft trees of `new` nodes each: parents, keys and values."""

    def __init__(self, rng, new, hkv, d, dtype, chain=False):
        self.indptr = starts(new)
        self.parent = np.concatenate([[-1 if i == 0 else i - 1 if chain else int(rng.integers(max(0, i - 6), i)) for i in range(n)]
                                      for n in new]).astype(np.int32)
        T = int(self.indptr[-1])
        self.k, self.v = (typed(rng.standard_normal((T, hkv, d)), dtype) for _ in range(2))


def run_tree(ada, q, trees, prefix, cache, dtype, scale, window, sinks, table=None):
    import torch
    T, hq, d = q.shape
    plen = np.asarray(prefix, np.int32)
    table = cache.table if table is None else table
    need = ada.adaserve_window_tree_attn_workspace_bytes(trees.indptr, plen, hq, cache.k.shape[1], d, PS, window, sinks, code(ada, dtype))
    rows = to_dev(q)
    out = torch.full(rows.shape, SENTINEL, dtype=rows.dtype, device="cuda")
    print("window tree nodes", T, "of", len(plen), "heads", hq, cache.k.shape[1], "D", d, dtype, "window", window, sinks,
          "workspace", need, flush=True)
    ada.adaserve_window_tree_attn(node_indptr=to_dev(trees.indptr), node_indptr_host=trees.indptr, parent=to_dev(trees.parent),
                                  q=rows, k_tree=to_dev(trees.k), v_tree=to_dev(trees.v), k_pages=to_dev(cache.k),
                                  v_pages=to_dev(cache.v), block_table=to_dev(table), prefix_len=to_dev(plen),
                                  prefix_len_host=plen, window=window, sinks=sinks, sm_scale=scale, out=out,
                                  workspace=workspace(need))
    torch.cuda.synchronize()
    return widen(back(out))


def seen_by_any(kind, n, c, window, sinks):
    """Positions 0 .. c - 1 that some row of a request with n new rows (nodes) sees: every row sees what the first does of the
    positions from the first one's window on."""
    first = c - n if kind == "prompt" else c - 1 if kind == "decode" else c
    at = np.arange(c)
    return (at < sinks) | (at > first - window)


def hide(rng, kind, cache, new, ctx, window, sinks):
    """Poisons (NaN) what no row of its request sees, and gives back the pages that hold nothing else: their entries become
    -1, another request's page, or numbers outside the pool."""
    cache.k, cache.v, table = cache.k.copy(), cache.v.copy(), cache.table.copy()
    nan = typed(np.full(1, np.nan, np.float32), "bf16")[0] if cache.k.dtype == np.uint16 else np.float32(np.nan)
    for r, (n, c) in enumerate(zip(new, ctx)):
        seen = seen_by_any(kind, n, c, window, sinks)
        for e in range(-(-c // PS)):
            mine = seen[e * PS:(e + 1) * PS]
            slots = np.flatnonzero(~mine)
            cache.k[cache.table[r, e], :, slots] = nan
            cache.v[cache.table[r, e], :, slots] = nan
            if not mine.any():
                table[r, e] = rng.choice([-1, int(rng.integers(0, cache.pages)), cache.pages + 5, -2 ** 31])
    cache.table = table
    return cache


# Half a step of the weights in the products with the values, and of a chunk's own output: prompts round weights to bf16,
# single tokens hold them in two bf16 parts; trees round the weights (of numerator and denominator) and split prefixes' outputs.
NUMERATOR = {"prompt": 2.0 ** -8, "decode": 2.0 ** -16, "tree": 2.0 ** -7}
DENOMINATOR = {"prompt": 0.0, "decode": 0.0, "tree": 2.0 ** -8}


def bound(kind, dtype, out, size, reach, keys, d):
    """The output's half step (of fp32: of the quotient, its operands and the join); the weights' roundings; and what moves a
    weight against the others: d products and sums of a score in fp32, 6 half steps of its scaling and exponent, 2^-21 of the
    exponential.  Sums run over at most `keys` terms, and 80 steps of joins and rescalings."""
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    num, den = (NUMERATOR[kind], DENOMINATOR[kind]) if dtype == "bf16" else (0.0, 0.0)
    moved = 2.0 ** -24 * (d + 6) * reach[..., None] + 2.0 ** -21 + 2.0 ** -24 * 2 * (keys + 80)
    return (step + den) * np.abs(out) + num * size + moved * (size + np.abs(out)) + 1e-30


def check(kind, dtype, got, expected, keys):
    out, size, reach = expected
    wrong = int((~np.isfinite(got)).sum())
    assert wrong == 0
    err, b = np.abs(got - out), bound(kind, dtype, out, size, reach, keys, out.shape[2])
    far = float((err / b).max(initial=0))
    assert far <= 1, (far, float(err.max()), np.argwhere(err > b)[:4].tolist())


def case(rng, kind, dtype, d, hq, hkv, new, ctx, window, sinks, whole=False):
    """Cache, trees and queries.  `whole`: values of whole numbers -8 .. 8 and queries of zeros, so that an output is the mean of
    the values that are seen: only its quotient is rounded."""
    cache = Cache(rng, ctx, hkv, d, dtype)
    trees = Trees(rng, new, hkv, d, dtype) if kind == "tree" else None
    T = len(ctx) if kind == "decode" else int(starts(new)[-1])
    q = np.zeros((T, hq, d)) if whole else rng.standard_normal((T, hq, d))
    if whole:
        cache.v = np.where(np.isnan(widen(cache.v)), cache.v, typed(rng.integers(-8, 9, cache.v.shape).astype(np.float32), dtype))
        if trees:
            trees.v = typed(rng.integers(-8, 9, trees.v.shape).astype(np.float32), dtype)
    cache = hide(rng, kind, cache, [1] * len(ctx) if kind == "decode" else new, ctx, window, sinks)
    return cache, trees, typed(q, dtype)


def run(ada, kind, dtype, cache, trees, q, new, ctx, scale, window, sinks, **kw):
    if kind == "prompt":
        return run_prompt(ada, q, new, ctx, cache, dtype, scale, window, sinks, **kw)
    if kind == "decode":
        return run_decode(ada, q, ctx, cache, dtype, scale, window, sinks, **kw)
    return run_tree(ada, q, trees, ctx, cache, dtype, scale, window, sinks, **kw)


def expected(kind, cache, trees, q, new, ctx, scale, window, sinks, table=None):
    table = cache.table if table is None else table
    if kind == "tree":
        return oracle.tree_attention(q, trees.indptr, trees.parent, trees.k, trees.v, cache.k, cache.v, table, ctx, scale,
                                     window, sinks)
    return oracle.paged_attention(q, starts([1] * len(ctx) if kind == "decode" else new), cache.k, cache.v, table, ctx, scale,
                                  window, sinks)


def mean_bound(kind, dtype, out, size):
    """Every weight is 1 and every sum exact: half a step of the output and of its quotient, and in trees of the chunks' own.
    The oracle's own sum is off by at most 2^-53 per term and operation of `size`, 2^-40 for the up to 1000 terms of four
    operations each: all of the difference where values cancel to 0."""
    half = (2.0 ** -8 + 2.0 ** -22) * np.abs(out) + (2.0 ** -8 * size if kind == "tree" else 0) if dtype == "bf16" \
        else 2.0 ** -21 * np.abs(out)
    return half + 2.0 ** -40 * size
