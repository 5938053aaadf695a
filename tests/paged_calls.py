"""Calls of prompt and single-token attention on given queries and caches, and
how far their results may be from fp64's, row by row."""
import numpy as np

from oracle import serving
from serving_inputs import PS, back, to_dev

SENTINEL = 77.0


def starts(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def run_prompt(ada, q, new, ctx, cache, dtype, scale, table=None, split=None, pad=0):
    """q [T, Hq, D] typed host rows.  `split`: whether the call has to split its keys."""
    import torch
    T, hq, d = q.shape
    indptr, ctx32 = starts(new), np.asarray(ctx, np.int32)
    table = cache.table if table is None else table
    code = ada.ADASERVE_BF16 if dtype == "bf16" else ada.ADASERVE_F32
    need = ada.adaserve_prompt_attn_workspace_bytes(indptr, ctx32, hq, cache.k.shape[1], d, PS, code)
    assert split is None or split == (need > 0)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    rows = to_dev(np.concatenate([q, np.zeros((pad, hq, d), q.dtype)]))
    out = torch.full(rows.shape, SENTINEL, dtype=rows.dtype, device="cuda")
    print("prompt rows", T, "requests", len(ctx32), "longest", int(ctx32.max(initial=0)), "workspace", need, flush=True)
    ada.adaserve_prompt_attn(token_indptr=to_dev(indptr), token_indptr_host=indptr, q=rows, k_pages=to_dev(cache.k),
                             v_pages=to_dev(cache.v), block_table=to_dev(table), context_len=to_dev(ctx32),
                             context_len_host=ctx32, sm_scale=scale, out=out, workspace=ws)
    torch.cuda.synchronize()
    got = serving.widen(back(out))
    assert (got[T:] == SENTINEL).all()
    return got[:T]


def run_decode(ada, q, ctx, cache, dtype, scale, most=None, table=None):
    import torch
    B, hq, d = q.shape
    ctx = np.asarray(ctx)
    table = cache.table if table is None else table
    most = int(ctx.max()) if most is None else most
    code = ada.ADASERVE_BF16 if dtype == "bf16" else ada.ADASERVE_F32
    need = ada.adaserve_decode_attn_workspace_bytes(B, most, hq, cache.k.shape[1], d, PS, code)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    rows = to_dev(q)
    out = torch.full(rows.shape, SENTINEL, dtype=rows.dtype, device="cuda")
    print("decode requests", B, "longest", int(ctx.max()), "workspace", need, flush=True)
    ada.adaserve_decode_attn(q=rows, k_pages=to_dev(cache.k), v_pages=to_dev(cache.v), block_table=to_dev(table),
                             context_len=to_dev(ctx.astype(np.int32)), max_context=most, sm_scale=scale, out=out, workspace=ws)
    torch.cuda.synchronize()
    return serving.widen(back(out))


def reach(q, indptr, cache, table, ctx, scale):
    """Per row of q [T, Hq, D]: the largest scale * sum |q_d k_d| over its request's keys."""
    q, k = np.abs(serving.widen(q)), np.abs(serving.widen(cache.k))
    T, hq, _ = q.shape
    P, hkv, G = k.shape[0], k.shape[1], q.shape[1] // k.shape[1]
    most = np.zeros((T, hq))
    for r, c in enumerate(ctx):
        place = np.arange(int(c))
        page = table[r][place // PS] if c else np.zeros(0, int)
        ok = (page >= 0) & (page < P)
        a, b = int(indptr[r]), int(indptr[r + 1])
        for h in range(hq):
            keys = k[page[ok], h // G, place[ok] % PS]
            keys = np.where(np.isfinite(keys), keys, 0)
            if b > a and len(keys):
                most[a:b, h] = (q[a:b, h] @ keys.T).max(1) * abs(scale)
    return most


# The weights' half step in the products with the values: prompts round them to
# bf16, single tokens hold them in two bf16 parts, 2^-8 of 2^-8.
WEIGHT = {("prompt", "bf16"): 2.0 ** -8, ("decode", "bf16"): 2.0 ** -16, ("prompt", "f32"): 0.0, ("decode", "f32"): 0.0}


def bound(kind, dtype, out, size, most, keys, d):
    """Half a step of the output (of fp32: of the quotient, its two operands and
    the join); of the weights in the numerator; and what moves a weight against
    the others: d fp32 products and sums of a score (half a step each of the
    largest sum of magnitudes, `most`), 6 for its scaling and exponent, and 2^-21
    of the exponential.  Sums run over at most a quarter of the keys (four waves),
    64 parts and 16 steps of joins, each once for a sum and once for a rescaling."""
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    moved = 2.0 ** -24 * (d + 6) * most[..., None] + 2.0 ** -21 + 2.0 ** -24 * 2 * (keys / 4 + 80)
    return step * np.abs(out) + WEIGHT[kind, dtype] * size + moved * (size + np.abs(out)) + 1e-30


def check(kind, got, q, new, ctx, cache, dtype, scale, table=None):
    """`got` against fp64 on the same inputs, for all rows."""
    table = cache.table if table is None else table
    indptr = starts(new)
    out, size, _ = serving.paged_attention(q, indptr, cache.k, cache.v, table, ctx, scale)
    most = reach(q, indptr, cache, table, ctx, scale)
    b = bound(kind, dtype, out, size, most, int(np.max(ctx, initial=0)), q.shape[2])
    assert np.isfinite(got).all(), int((~np.isfinite(got)).sum())
    err = np.abs(got - out)
    assert (err <= b).all(), (float((err / b).max()), float(err.max()))
