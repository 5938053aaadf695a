"""Attention over a window and sinks of thousands of rows in fp64, a request's scores of one head at a time, and the bound
of means whose prefixes are split."""
import numpy as np
import torch

from oracle.serving import widen
from paged_calls import starts
from serving_inputs import PS


def paths(parent):
    """[n, n]: node i's root-to-node path, of one tree's parents."""
    on = np.eye(len(parent), dtype=bool)
    for i, p in enumerate(parent):
        if p >= 0:
            on[i] |= on[p]
    return on


def seen_positions(kind, n, c, window, sinks, parent=None):
    """[n, keys]: which of its request's keys, the c cached ones and behind them a tree's n nodes, a row sees."""
    at = np.arange(c)
    pos = c - n + np.arange(n)
    on = np.zeros((n, 0), bool)
    if kind == "tree":
        on = paths(parent)
        pos = c + on.sum(1) - 1
        at = np.concatenate([at, pos])
    before = at[None, :] <= pos[:, None]
    if kind == "tree":
        before[:, c:] = on
    return before & ((at[None, :] > pos[:, None] - window) | (at[None, :] < sinks))


def _rows(q, k, v, seen, scale):
    """One head's rows: (output, sum of weight * |value|, largest sum |q_d k_d|)."""
    some = torch.as_tensor(seen.any(0), device=q.device)[:, None]
    k, v = torch.where(some, k, 0.0), torch.where(some, v, 0.0)
    hidden = ~torch.as_tensor(seen, device=q.device)
    z = (q @ k.T * scale).masked_fill_(hidden, -torch.inf)
    top = z.amax(1, keepdim=True)
    w = (z - torch.where(top == -torch.inf, 0.0, top)).exp_()
    total = w.sum(1, keepdim=True)
    w /= torch.where(total == 0, 1.0, total)
    reach = (q.abs() @ k.abs().T * abs(scale)).masked_fill_(hidden, 0.0).amax(1)
    return w @ v, w @ v.abs(), reach


def expected(kind, cache, trees, q, new, ctx, scale, window, sinks, device="cuda"):
    """As window_calls.expected, of prompts and trees: dense, on a device."""
    t64 = lambda x: torch.as_tensor(np.asarray(widen(x), np.float64), device=device)  # noqa: E731
    indptr, rows, kp, vp = starts(new), t64(q), t64(cache.k), t64(cache.v)
    T, hq, d = rows.shape
    group = hq // kp.shape[1]
    out, size = torch.zeros_like(rows), torch.zeros_like(rows)
    reach = torch.zeros(T, hq, dtype=torch.float64, device=device)
    for r, (n, c) in enumerate(zip(new, ctx)):
        if n == 0:
            continue
        a, b = int(indptr[r]), int(indptr[r + 1])
        at = np.arange(c)
        page = cache.table[r][at // PS].astype(np.int64)
        there = torch.as_tensor((page >= 0) & (page < cache.pages), device=device)[:, None]
        page, slot = (torch.as_tensor(x, device=device) for x in (np.clip(page, 0, cache.pages - 1), at % PS))
        seen = seen_positions(kind, n, c, window, sinks, trees.parent[a:b] if kind == "tree" else None)
        for h in range(hq):
            g = h // group
            k, v = (torch.where(there, x[page, g, slot], 0.0) for x in (kp, vp))
            if kind == "tree":
                k, v = torch.cat([k, t64(trees.k[a:b, g])]), torch.cat([v, t64(trees.v[a:b, g])])
            out[a:b, h], size[a:b, h], reach[a:b, h] = _rows(rows[a:b, h], k, v, seen, scale)
    return tuple(x.cpu().numpy() for x in (out, size, reach))


def split_mean_bound(out, size):
    """bf16 means (every weight 1, every sum of a chunk exact) whose keys are split, the chunks' outputs held in fp32: half a
    step of the output and 2^-22 of its quotient; of a chunk's output two half steps, and two of the sum at each of at most
    14 chunks, all of at most `size`.  The rest is the reference's own, as in window_calls.mean_bound."""
    return (2.0 ** -8 + 2.0 ** -22) * np.abs(out) + (30 * 2.0 ** -24 + 2.0 ** -40) * size
