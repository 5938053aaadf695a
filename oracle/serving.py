"""TEST INFRASTRUCTURE ONLY: the serving operators in fp64, from their
definitions (numpy, plain loops over requests and heads).  Shares no code with
the HIP library."""
from __future__ import annotations

import numpy as np

UNIT = 4294967296.0   # 2^32: whole units of a token's mass


def widen(a) -> np.ndarray:
    """fp64 values of an array; uint16 arrays are bf16 bit patterns."""
    a = np.asarray(a)
    if a.dtype == np.uint16:
        return (a.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return a.astype(np.float64)


def rope(x, pos, inv_freq, interleaved=False):
    """x [T, H, D] rotated at positions pos [T] (fp64 result)."""
    y = widen(x).copy()
    inv = np.asarray(inv_freq, np.float32).astype(np.float64)
    h = inv.size
    angle = np.asarray(pos, np.float64)[:, None] * inv[None, :]
    c, s = np.cos(angle)[:, None, :], np.sin(angle)[:, None, :]
    first = slice(0, 2 * h, 2) if interleaved else slice(0, h)
    second = slice(1, 2 * h, 2) if interleaved else slice(h, 2 * h)
    a, b = y[..., first].copy(), y[..., second].copy()
    y[..., first] = a * c - b * s
    y[..., second] = a * s + b * c
    return y


def append_places(token_indptr, prefix_len, block_table, num_pages, page_size, num_tokens):
    """Per token: request (-1: none), cache place, page (-1: not stored); and the new lengths."""
    T, B = num_tokens, len(prefix_len)
    req, place, page = np.full(T, -1), np.zeros(T, np.int64), np.full(T, -1)
    new = np.array(prefix_len, np.int64)
    for r in range(B):
        L, whole = int(prefix_len[r]), True
        for t in range(max(int(token_indptr[r]), 0), min(int(token_indptr[r + 1]), T)):
            req[t], place[t] = r, L + t - int(token_indptr[r])
            if L < 0:
                continue
            e = place[t] // page_size
            p = int(block_table[r, e]) if e < block_table.shape[1] else -1
            if 0 <= p < num_pages:
                page[t] = p
                new[r] += whole
            else:
                whole = False
    return req, place, page, new


def attend(q, keys, values, sm_scale, visible):
    """q [n, D] over keys, values [c, D]; row i sees the first visible[i] of them.
    Returns (output, sum of weight * |value|, largest sum |q_d k_d| * |scale|)."""
    n, c = q.shape[0], keys.shape[0]
    out, size = np.zeros_like(q), np.zeros_like(q)
    reach = 0.0
    if n and c:
        see = np.arange(c)[None, :] < np.asarray(visible)[:, None]
        z = np.where(see, np.where(see, q @ np.where(np.isfinite(keys), keys, 0).T, 0) * sm_scale, -np.inf)
        m = z.max(1, keepdims=True)
        w = np.exp(z - np.where(np.isfinite(m), m, 0))
        l = w.sum(1, keepdims=True)
        w = np.divide(w, l, out=np.zeros_like(w), where=l > 0)
        v = np.where(np.isfinite(values), values, 0)
        out, size = w @ v, w @ np.abs(v)
        reach = float((np.abs(q).max(0, initial=0) @ np.abs(np.where(np.isfinite(keys), keys, 0)).max(0, initial=0)) * abs(sm_scale))
    return out, size, reach


def paged_attention(q, token_indptr, k_pages, v_pages, block_table, context_len, sm_scale):
    """Causal attention of packed rows q [T, Hq, D] over paged keys, values
    [P, Hkv, page_size, D]: row i of request r's n at position c - n + i.
    Returns (output, sum of weight * |value|, largest |score| bound)."""
    q, kp, vp = widen(q), widen(k_pages), widen(v_pages)
    T, Hq, D = q.shape
    P, Hkv, ps, _ = kp.shape
    G = Hq // Hkv
    out, size, reach = np.zeros_like(q), np.zeros_like(q), 0.0
    for r in range(len(context_len)):
        a, b, c = int(token_indptr[r]), int(token_indptr[r + 1]), int(context_len[r])
        n = b - a
        place = np.arange(c)
        page = block_table[r][place // ps] if c else np.zeros(0, int)
        ok = (page >= 0) & (page < P)
        visible = np.maximum(c - n + np.arange(n) + 1, 0)
        for g in range(Hkv):
            k = np.where(ok[:, None], kp[np.where(ok, page, 0), g, place % ps], 0)
            v = np.where(ok[:, None], vp[np.where(ok, page, 0), g, place % ps], 0)
            for h in range(g * G, (g + 1) * G):
                o, s, z = attend(q[a:b, h], k, v, sm_scale, visible)
                out[a:b, h], size[a:b, h], reach = o, s, max(reach, z)
    return out, size, reach


def sample_row(x, temperature, top_k, top_p, min_p, u):
    """The token of one row of logits (fp32 parameters), -1 where the row or its parameters are no distribution."""
    x = widen(x) + 0.0
    t, p, m, u = (np.float64(np.float32(v)) for v in (temperature, top_p, min_p, u))
    if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any():
        return -1
    if not (0 <= t < np.inf) or np.isnan(p) or np.isnan(m) or np.isnan(u):
        return -1
    order = np.lexsort((np.arange(x.size), -x))
    if t == 0 or m > 1:
        return int(order[0])
    mass = [int(v) for v in np.rint(np.exp((x - x.max()) / t) * UNIT)]
    if 1 <= top_k < x.size:
        order = order[:top_k]
    if p < 1:
        whole = float(sum(mass[i] for i in order))
        kept, before = [], 0
        for i in order:
            if kept and not float(before) < p * whole:
                break
            kept.append(i)
            before += mass[i]
        order = kept
    order = sorted(i for i in order if mass[i] >= m * UNIT)
    target = max(u, 0.0) * float(sum(mass[i] for i in order))
    upto, last = 0, -1
    for i in order:
        upto += mass[i]
        if mass[i]:
            last = int(i)
            if float(upto) > target:
                break
    return last


def sample(logits, vocab, temperature=None, top_k=None, top_p=None, min_p=None, u=None):
    rows = len(logits)
    full = lambda a, v: np.full(rows, v) if a is None else a
    t, k, p, m = full(temperature, 1.0), full(top_k, 0), full(top_p, 1.0), full(min_p, 0.0)
    return np.array([sample_row(logits[i][:vocab], t[i], int(k[i]), p[i], m[i], u[i]) for i in range(rows)], np.int32)
