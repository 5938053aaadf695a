"""Caches on which a key too few, a key too many or a page in the wrong place shows in the result, however long they are."""
import numpy as np

from oracle import serving
from paged_calls import starts
from serving_inputs import PS, Cache, typed


def counted(rng, ctx, hkv, d, dtype):
    """Values are whole numbers of -8 .. 8 and queries (zeros) see all keys alike: a row's output is the mean of the values it
    sees, every weight is 1 and every sum exact in fp32, so that only the quotient is rounded."""
    c = Cache(rng, ctx, hkv, d, dtype)
    whole = typed(rng.integers(-8, 9, c.v.shape).astype(np.float32), dtype)
    c.v = np.where(np.isnan(serving.widen(c.v)), c.v, whole)
    return c


def means(cache, new, ctx, hq, table=None):
    """The outputs of zero queries, exactly: [rows, hq, D]."""
    table = cache.table if table is None else table
    v = serving.widen(cache.v)
    hkv, d = v.shape[1], v.shape[3]
    rows = []
    for r, (n, c) in enumerate(zip(new, ctx)):
        place = np.arange(c)
        x = v[table[r][place // PS], :, place % PS] if c else np.zeros((0, hkv, d))
        upto = np.concatenate([np.zeros((1, hkv, d)), np.cumsum(x, 0)])
        seen = np.maximum(c - n + np.arange(n) + 1, 0)
        rows.append(upto[seen] / np.maximum(seen, 1)[:, None, None])
    return np.repeat(np.concatenate(rows), hq // hkv, 1)


def mean_bound(dtype, out):
    """Half a step of the output; of fp32 of its quotient: a reciprocal and a product (one each), or a division."""
    return (2.0 ** -8 + 2.0 ** -22 if dtype == "bf16" else 2.0 ** -22) * np.abs(out)


def places(rng, c):
    """Where something begins or ends in c keys: the first and the last, and beside multiples of what pages, blocks, waves
    and windows of page ids hold."""
    at = [0, c - 1]
    for step in (16, 32, 64, 128, 512, 1024, 2048):
        m = step * int(rng.integers(0, c // step + 1))
        at += [m - 1, m, c // step * step - 1, c // step * step]
    return np.array([p for p in at if 0 <= p < c] + list(rng.integers(0, c, 4)))


def pointed(rng, new, ctx, hq, hkv, d, dtype):
    """Queries that are four times one key that they see, at a place where something ends: nearly all of the weight is its."""
    c = Cache(rng, ctx, hkv, d, dtype)
    keys = serving.widen(c.k)
    q = rng.standard_normal((int(starts(new)[-1]), hq, d))
    for r, (n, length) in enumerate(zip(new, ctx)):
        at = places(rng, length) if length else np.zeros(0, int)
        for i in range(n):
            seen = length - n + i + 1
            if seen <= 0:
                continue
            mine = np.concatenate([[seen - 1, 0], at[at < seen]])
            # the last key and the first for two heads, any of them for the others
            pick = mine[np.where(np.arange(hq) < 2, np.arange(hq), rng.integers(0, len(mine), hq))]
            q[starts(new)[r] + i] = 4 * keys[c.table[r][pick // PS], np.arange(hq) // (hq // hkv), pick % PS]
    return c, typed(q, dtype)
