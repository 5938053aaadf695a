"""TEST INFRASTRUCTURE ONLY: attention over a window and sinks, and the pages of
the cache, from their definitions (numpy, plain loops).  Shares no code with the
HIP library."""
from __future__ import annotations

import numpy as np

from .serving import widen


def sees(row_pos, key_pos, window, sinks):
    """Which positions key_pos [c] a row at row_pos sees."""
    key_pos = np.asarray(key_pos)
    return (key_pos <= row_pos) & ((key_pos > row_pos - window) | (key_pos < sinks))


def attend_rows(q, keys, values, seen, sm_scale):
    """q [n, D] over keys, values [c, D], row i over seen[i]: (output, sum of weight * |value|, largest sum |q_d k_d| per row);
    what no row sees may hold anything."""
    any_row = seen.any(0)
    k, v = np.where(any_row[:, None], keys, 0), np.where(any_row[:, None], values, 0)
    n, d = q.shape
    out, size, reach = np.zeros((n, d)), np.zeros((n, d)), np.zeros(n)
    for i in range(n):
        at = np.flatnonzero(seen[i])
        if at.size == 0:
            continue
        z = k[at] @ q[i] * sm_scale
        w = np.exp(z - z.max())
        w /= w.sum()
        out[i], size[i] = w @ v[at], w @ np.abs(v[at])
        reach[i] = (np.abs(k[at]) @ np.abs(q[i])).max() * abs(sm_scale)
    return out, size, reach


def _cached(pool, table_row, places, g, ps):
    """Rows of kv-head g at the places of a request; zeros where its table names no page."""
    rows = np.zeros((len(places), pool.shape[3]))
    for i, t in enumerate(places):
        e = t // ps
        p = int(table_row[e]) if e < len(table_row) else -1
        if 0 <= p < pool.shape[0]:
            rows[i] = pool[p, g, t % ps]
    return rows


def paged_attention(q, token_indptr, k_pages, v_pages, block_table, context_len, sm_scale, window, sinks):
    """Rows q [T, Hq, D] at positions c - n + i of their requests' paged caches: (output, size, reach [T, Hq])."""
    q, kp, vp = widen(q), widen(k_pages), widen(v_pages)
    T, Hq, D = q.shape
    P, Hkv, ps, _ = kp.shape
    G = Hq // Hkv
    out, size, reach = np.zeros_like(q), np.zeros_like(q), np.zeros((T, Hq))
    for r in range(len(context_len)):
        a, b, c = int(token_indptr[r]), int(token_indptr[r + 1]), int(context_len[r])
        pos = c - (b - a) + np.arange(b - a)
        seen = np.stack([sees(p, np.arange(c), window, sinks) for p in pos]) if b > a else np.zeros((0, c), bool)
        used = np.flatnonzero(seen.any(0))
        for g in range(Hkv):
            k, v = _cached(kp, block_table[r], used, g, ps), _cached(vp, block_table[r], used, g, ps)
            for h in range(g * G, (g + 1) * G):
                out[a:b, h], size[a:b, h], reach[a:b, h] = attend_rows(q[a:b, h], k, v, seen[:, used], sm_scale)
    return out, size, reach


def tree_attention(q, node_indptr, parent, k_tree, v_tree, k_pages, v_pages, block_table, prefix_len, sm_scale, window, sinks):
    """Nodes q [T, Hq, D] at positions L + depth over the prefix and their root-to-node paths."""
    q, kt, vt, kp, vp = (widen(x) for x in (q, k_tree, v_tree, k_pages, v_pages))
    T, Hq, D = q.shape
    P, Hkv, ps, _ = kp.shape
    G = Hq // Hkv
    out, size, reach = np.zeros_like(q), np.zeros_like(q), np.zeros((T, Hq))
    for r in range(len(prefix_len)):
        a, b, L = int(node_indptr[r]), int(node_indptr[r + 1]), int(prefix_len[r])
        paths = []
        for i in range(b - a):
            p = int(parent[a + i])
            paths.append(([] if p < 0 else paths[p]) + [i])
        pos = np.array([L + len(p) - 1 for p in paths], np.int64)
        seen = np.zeros((b - a, L + b - a), bool)
        for i, path in enumerate(paths):
            seen[i, :L] = sees(pos[i], np.arange(L), window, sinks)
            for n in path:
                seen[i, L + n] = sees(pos[i], pos[n], window, sinks)
        used = np.flatnonzero(seen[:, :L].any(0))
        cols = np.concatenate([used, np.arange(L, L + b - a)])
        for g in range(Hkv):
            k = np.concatenate([_cached(kp, block_table[r], used, g, ps), kt[a:b, g]])
            v = np.concatenate([_cached(vp, block_table[r], used, g, ps), vt[a:b, g]])
            for h in range(g * G, (g + 1) * G):
                out[a:b, h], size[a:b, h], reach[a:b, h] = attend_rows(q[a:b, h], k, v, seen[:, cols], sm_scale)
    return out, size, reach


def _inside(p, refs):
    return 0 <= p < len(refs)


def _free(refs):
    """The free pages, the lowest first."""
    return iter([p for p in range(len(refs)) if refs[p] <= 0])


def update_pages(context_len, need_len, window, sinks, ps, table, refs):
    """(new table, new references, capacity; None without need_len)."""
    table, refs = [[int(p) for p in row] for row in table], [int(n) for n in refs]
    for c, row in zip(context_len, table):
        for e in range(len(row)):
            wanted = [j for j in range(e * ps, (e + 1) * ps) if j < sinks or window == 0 or j > int(c) - window]
            if c >= 0 and wanted:
                continue
            if _inside(row[e], refs):
                refs[row[e]] -= 1
            row[e] = -1
    capacity, free = [], _free(refs)
    for r, row in enumerate(table if need_len is not None else []):
        c, need = int(context_len[r]), int(need_len[r])
        if c < 0:
            capacity.append(0)
            continue
        for e in range(len(row)):
            # (an entry whose first position is from c on and below need)
            if c <= e * ps < need and not _inside(row[e], refs):
                p = next(free, None)
                if p is not None:
                    row[e], refs[p] = p, 1
        at = c
        while at < need and at // ps < len(row) and _inside(row[at // ps], refs):
            at += 1
        capacity.append(need if need <= c else at)
    shape = (len(table), len(table[0]) if table else 0)
    return np.array(table, np.int32).reshape(shape), np.array(refs, np.int32), \
        np.array(capacity, np.int32) if need_len is not None else None


def fork_pages(source, context_len, ps, table, refs):
    """(new table, new lengths, new references, copy_src, copy_dst)."""
    refs = [int(n) for n in refs]
    stride = table.shape[1]
    for row in table:
        for p in row:
            if _inside(p, refs):
                refs[p] -= 1
    new, lens, first = [], [], {}
    for r, s in enumerate(source):
        row, c = [-1] * stride, 0
        if 0 <= s < len(table):
            c = min(max(int(context_len[s]), 0), stride * ps)
            keep = stride if s not in first else c // ps
            row[:keep] = [int(p) for p in table[s][:keep]]
            first.setdefault(int(s), r)
        for p in row:
            if _inside(p, refs):
                refs[p] += 1
        new.append(row)
        lens.append(c)
    src, dst, free = [-1] * len(new), [-1] * len(new), _free(refs)
    for r, s in enumerate(source):
        e = lens[r] // ps
        if not 0 <= s < len(table) or first[int(s)] == r or lens[r] % ps == 0 or not _inside(table[s][e], refs):
            continue
        p = next(free, None)
        if p is None:
            lens[r] = e * ps
        else:
            new[r][e], refs[p], src[r], dst[r] = p, 1, int(table[s][e]), p
    i32 = lambda x: np.array(x, np.int32)  # noqa: E731
    return i32(new).reshape(len(new), stride), i32(lens), i32(refs), i32(src), i32(dst)


def compact_pages(table, refs):
    """(new table, new references, new places, move_src, move_dst, counts)."""
    P = len(refs)
    used = [p for p in range(P) if refs[p] > 0]
    place, src, dst = {}, [], []
    holes = (p for p in range(len(used)) if refs[p] <= 0)
    for p in used:
        place[p] = p
        if p >= len(used):
            place[p] = next(holes)
            src.append(p)
            dst.append(place[p])
    new_refs = np.zeros(P, np.int32)
    for p, q in place.items():
        new_refs[q] = refs[p]
    new = np.array([[place.get(int(p), -1) if _inside(p, refs) else int(p) for p in row] for row in table],
                   np.int32).reshape(table.shape)
    fill = [-1] * (P - len(src))
    return new, new_refs, np.array([place.get(p, -1) for p in range(P)], np.int32), np.array(src + fill, np.int32), \
        np.array(dst + fill, np.int32), np.array([len(used), len(src)], np.int32)
