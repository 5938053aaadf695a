"""Serving over a window: attention that sees a window of the newest keys and a few first ones, and the pages of its cache.

A case is one call, or one that another completes:

* ``prompt``   causal attention of packed prompts, or chunks of them, whose rows see the window's keys and the sinks;
* ``decode``   the same of one new token per request;
* ``tree``     the same of the nodes of draft trees, over the cached prefix and their root-to-node paths;
* ``update``   one step's bookkeeping: pages that have left the window are freed, pages for the next tokens are taken;
* ``fork``     rows of the cache go over to other rows (beams to their children, a prompt to its samples) by sharing
               pages, and the partly filled ones are copied;
* ``compact``  the pages in use move to the front of the pool, tables and contents.

Lengths and page places come from the case (``sizes``) and ``prepare``'s seed; what no row sees any more has no page.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
PAGE = 16
BLOCK = 256          # rows that the plain form of prompts takes together

# The dearest drawn case stays within these (one pass of the largest listed ones).
MOST_PROMPT_FLOPS = 3.3e11
MOST_PROMPT_FLOPS_F32 = 3e10
MOST_SCORES = 1.2e9          # padded scores of the plain form
MOST_CACHE_BYTES = 5.1e8       # what a call has to read of the cache
MOST_POOL_BYTES = 1.5e9
MOST_ENTRIES = 600000        # of a block table
MOST_COPIED = 2.7e8


def listed():
    chat = {"hq": 32, "hkv": 8, "dim": 128, "dtype": "bf16"}
    big = {"hq": 64, "hkv": 8, "dim": 128, "dtype": "bf16"}
    return [
        # Eight ragged prompts of chat requests at once, longer than the window: the usual prefill of one layer.
        {"name": "prompt_8b", "kind": "prompt", "requests": 8, "new_lo": 600, "new_hi": 5000, "len_lo": 0, "len_hi": 0,
         "window": 1024, "sinks": 4, "sizes": 1, **chat},
        # fp32 chunks of three prompts over what is cached of them, head dimension 64, as a numerics run makes them.
        {"name": "prompt_chunks_f32", "kind": "prompt", "requests": 3, "new_lo": 1, "new_hi": 700, "len_lo": 100,
         "len_hi": 2500, "window": 512, "sinks": 16, "hq": 8, "hkv": 8, "dim": 64, "dtype": "f32", "sizes": 2},
        # The next token of an idle server's only user, far into a long chat: latency.
        {"name": "decode_one_user", "kind": "decode", "requests": 1, "len_lo": 20001, "len_hi": 20001, "window": 4096,
         "sinks": 4, "sizes": 3, **chat},
        # Every request of a full server with the 70B shape's heads, ragged, long chats and new ones.
        {"name": "decode_70b", "kind": "decode", "requests": 64, "len_lo": 0, "len_hi": 16384, "window": 2048, "sinks": 4,
         "sizes": 4, **big},
        # Draft trees of 16 requests far into long texts, verified in one pass.
        {"name": "tree_8b", "kind": "tree", "requests": 16, "new_lo": 16, "new_hi": 64, "len_lo": 3000, "len_hi": 20000,
         "window": 2048, "sinks": 4, "sizes": 5, **chat},
        # Draft trees in fp32 with a window that is shorter than their prefixes by little, head dimension 64.
        {"name": "tree_f32", "kind": "tree", "requests": 4, "new_lo": 8, "new_hi": 40, "len_lo": 60, "len_hi": 900,
         "window": 255, "sinks": 8, "hq": 16, "hkv": 4, "dim": 64, "dtype": "f32", "sizes": 6},
        # A decoding step of a small server: now and then a page leaves a window, now and then one is taken.
        {"name": "update_step", "kind": "update", "requests": 24, "stride": 256, "pages": 4096, "len_hi": 4000, "grow_lo": 1,
         "grow_hi": 1, "window": 1024, "sinks": 4, "over": 0.0, "fill": 0.6, "lag": 1},
        # A large server's step: prompts that arrive take hundreds of pages each, finished requests give theirs back.
        {"name": "update_arrivals", "kind": "update", "requests": 250, "stride": 2048, "pages": 100003, "len_hi": 30000,
         "grow_lo": 1, "grow_hi": 6000, "window": 4096, "sinks": 4, "over": 0.15, "fill": 0.7, "lag": 128},
        # Beam search: 16 requests of 8 beams, whose children take over their caches.
        {"name": "fork_beams", "kind": "fork", "sources": 128, "requests": 128, "beams": 8, "stride": 40, "pages": 3200,
         "len_lo": 50, "len_hi": 600, "hkv": 8, "dim": 128, "dtype": "bf16", "layers": 1},
        # Two prompts go on as five samples each, fp32.
        {"name": "fork_samples", "kind": "fork", "sources": 2, "requests": 10, "beams": 0, "stride": 130, "pages": 300,
         "len_lo": 700, "len_hi": 2000, "hkv": 4, "dim": 64, "dtype": "f32", "layers": 2},
        # A small pool in which little is left to move.
        {"name": "compact_small", "kind": "compact", "requests": 8, "stride": 60, "pages": 600, "used": 0.9, "hkv": 2,
         "dim": 64, "dtype": "f32", "layers": 1},
        # A server's pool, half empty after its busy hours, before memory is handed to something else.
        {"name": "compact_server", "kind": "compact", "requests": 100, "stride": 40, "pages": 8000, "used": 0.45, "hkv": 8,
         "dim": 128, "dtype": "bf16", "layers": 1},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choices(["prompt", "decode", "tree", "update", "fork", "compact"], [4, 3, 3, 2, 2, 1])[0]
    c = {"kind": kind}
    if kind == "update":
        c["requests"] = _log_int(rng, 1, 512)
        c["stride"] = _log_int(rng, 1, max(1, min(4096, MOST_ENTRIES // c["requests"])))
        c["pages"] = _log_int(rng, 1, 200000)
        c["len_hi"] = rng.randint(0, c["stride"] * PAGE)
        c["grow_lo"], c["grow_hi"] = rng.choice([(1, 1), (1, 64), (0, _log_int(rng, 1, 8000))])
        c["window"] = rng.choice([0, _log_int(rng, 1, 16384), _log_int(rng, 1, 16384)])
        c["sinks"] = rng.choice([0, 4, _log_int(rng, 1, 100)])
        c["over"], c["fill"] = rng.choice([0.0, 0.2]), rng.choice([0.3, 0.7, 0.95, 1.0])
        c["lag"] = rng.choice([1, 17, 300])
        return c
    c["dtype"] = "f32" if rng.random() < 0.25 else "bf16"
    c["dim"] = 128 if rng.random() < 0.7 else 64
    if kind in ("fork", "compact"):
        c["hkv"], c["layers"] = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 3])
        page = 2 * c["hkv"] * PAGE * c["dim"] * _size(c) * c["layers"]     # bytes of its keys and values
        if kind == "fork":
            c["beams"] = rng.choice([0, 2, 4, 8])
            c["sources"] = _log_int(rng, 1, 256)
            c["requests"] = c["sources"] if c["beams"] else _log_int(rng, 1, 256)
            if c["beams"]:
                c["sources"] = c["requests"] = max(c["beams"], c["sources"] // c["beams"] * c["beams"])
            while c["requests"] * page > MOST_COPIED / 2:
                c["hkv"], page = c["hkv"] // 2, page // 2
            c["stride"] = _log_int(rng, 2, max(2, min(600, int(MOST_POOL_BYTES / page / c["sources"] / 1.5))))
            c["pages"] = _fork_pages(c)
            c["len_hi"] = rng.randint(1, c["stride"] * PAGE)
            c["len_lo"] = rng.randint(0, c["len_hi"])
        else:
            c["pages"] = _log_int(rng, 1, int(min(16000, MOST_COPIED / page)))
            c["requests"] = _log_int(rng, 1, 128)
            c["stride"] = max(1, c["pages"] // c["requests"] + rng.randint(0, 9))
            c["used"] = rng.choice([0.0, 0.1, 0.5, 0.9, 1.0])
        return c
    c["hq"], c["hkv"] = rng.choice([(32, 8), (64, 8), (16, 2), (8, 8), (16, 4), (32, 2), (16, 16), (4, 2), (28, 4), (6, 2)])
    c["window"] = _log_int(rng, 1, 8192)
    c["sinks"] = rng.choice([0, 1, 4, 4, 16, _log_int(rng, 1, 100)])
    c["sizes"] = rng.randrange(1 << 20)
    c["requests"] = _log_int(rng, 1, 64)
    c["len_hi"] = rng.choice([0, _log_int(rng, 1, 32768), _log_int(rng, 1, 32768)])
    if kind == "decode":
        c["len_hi"] = max(1, c["len_hi"])
    c["len_lo"] = rng.randint(0, c["len_hi"])
    if kind == "tree":
        c["new_hi"] = _log_int(rng, 1, 128)
        c["new_lo"] = rng.randint(1, c["new_hi"])
    elif kind == "prompt":
        c["new_hi"] = _log_int(rng, 1, 8192)
        c["new_lo"] = rng.randint(0, c["new_hi"])
    most = MOST_PROMPT_FLOPS if c["dtype"] == "bf16" else MOST_PROMPT_FLOPS_F32
    while True:
        w = work(c)
        keys = min(c["window"], c["len_hi"] + c.get("new_hi", 0)) + c["sinks"]
        blocks = c["requests"] * (1 if kind != "prompt" else -(-c["new_hi"] // BLOCK))
        rows = 1 if kind == "decode" else c["new_hi"] if kind == "tree" else BLOCK
        scores = blocks * rows * c["hq"] * (keys + BLOCK)
        band = blocks * (keys + BLOCK) * c["hkv"] * c["dim"] * 8
        if w["bytes"] <= MOST_CACHE_BYTES and w["flops"] <= most and scores <= MOST_SCORES and band <= 8e9:
            for at in ("new_lo", "len_lo"):
                if at in c and (kind != "tree" or at == "new_lo"):
                    before, new = _lens(c)
                    c[at] = max(c[at], int((before if kind == "decode" else new).sum() == 0))
                    break
            return c
        if c["requests"] > 1:
            c["requests"] = c["requests"] * 3 // 4
        elif kind != "prompt" or c["new_hi"] < 64:
            c["window"] = max(1, c["window"] // 2)
        else:
            c["new_hi"] = c["new_hi"] * 3 // 4
            c["new_lo"] = min(c["new_lo"], c["new_hi"])


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _fork_pages(case):
    """A pool with room for every source's row and, mostly, for the copies."""
    return case["sources"] * case["stride"] + case["requests"] // 2 + 1


def _lens(case):
    """Cached tokens before the call and new tokens (nodes), per request."""
    g = np.random.Generator(np.random.PCG64(case["sizes"]))
    before = g.integers(case["len_lo"], case["len_hi"] + 1, case["requests"])
    if case["kind"] == "decode":
        return before, np.ones_like(before)
    new = g.integers(case["new_lo"], case["new_hi"] + 1, case["requests"])
    return before, new


def _seen(pos, window, sinks):
    """Keys that a row at position `pos` (-1: none) sees."""
    pos = np.asarray(pos, np.float64)
    far = np.maximum(pos + 1 - window, 0)              # the first key of its window
    return np.where(pos < 0, 0, pos + 1 - far + np.minimum(sinks, far))


def work(case):
    kind = case["kind"]
    if kind in ("update", "fork", "compact"):
        entries = 4.0 * case["stride"] * case["requests"]
        refs = 4.0 * case["pages"]
        if kind == "update":
            return {"bytes": 2 * entries + 2 * refs + 12 * case["requests"], "flops": 2 * case["stride"] * case["requests"]}
        page = 2 * case["hkv"] * PAGE * case["dim"] * _size(case) * case["layers"]
        if kind == "fork":
            copies = max(0.0, case["requests"] - case["sources"] * 0.64) if not case["beams"] else case["requests"] * 0.35
            return {"bytes": 4.0 * case["stride"] * case["sources"] + entries + 2 * refs + 2 * copies * page,
                    "flops": case["stride"] * (case["sources"] + case["requests"])}
        moves = case["pages"] * case["used"] * (1 - case["used"])
        return {"bytes": 2 * entries + 3 * refs + 2 * moves * page, "flops": 2 * case["pages"]}
    s, n = _size(case), case["requests"]
    before, new = (a.astype(np.float64) for a in _lens(case))
    hq, hkv, d, w, sinks = case["hq"], case["hkv"], case["dim"], case["window"], case["sinks"]
    if kind == "decode":
        keys = float(_seen(before - 1, w, sinks).sum())
        return {"bytes": 2 * keys * hkv * d * s + 2 * n * hq * d * s + keys / PAGE * 4, "flops": 4 * keys * hq * d}
    rows = float(new.sum())
    if kind == "tree":
        keys = float(_seen(before - 1, w, sinks).sum())
        pairs = float((new * _seen(before - 1, w, sinks)).sum()) + rows * 4
        return {"bytes": 2 * (keys + rows) * hkv * d * s + 2 * rows * hq * d * s, "flops": 4 * pairs * hq * d}
    first = np.maximum(before + 1 - w, 0)              # the first key that a request's first row sees
    ctx = float(((before + new - first) + np.minimum(sinks, first))[new > 0].sum())
    pairs = sum(float(_seen(np.arange(b, b + m), w, sinks).sum()) for b, m in zip(before, new))
    return {"bytes": 2 * ctx * hkv * d * s + 2 * rows * hq * d * s, "flops": 4 * pairs * hq * d}


def _rng(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device=DEVICE)


def prepare(case, seed):
    if case["kind"] in ("update", "fork", "compact"):
        return _prepare_pages(case, seed)
    g = _rng(seed)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE).to(dtype)

    kind, n = case["kind"], case["requests"]
    before, new = _lens(case)
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    end = before + new if kind == "prompt" else before
    # the first position whose window counts: of the first row of a prompt, of the token, of the root
    at = before if kind != "decode" else np.maximum(before - 1, 0)
    wide = max(1, int((-(-end // PAGE)).max()))
    place = np.arange(wide)[None, :] * PAGE
    live = (place < end[:, None]) & ((place < case["sinks"]) | (place + PAGE > (at + 1 - case["window"])[:, None]))
    total = int(live.sum())
    pool = total + 4
    perm = torch.randperm(pool, generator=g, device=DEVICE).cpu().numpy()
    table = np.full((n, wide), -1)
    table[live] = perm[:total]          # (the pages before have been freed)
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    t = int(indptr[-1])
    s = {"case": case, "block_table": _i32(table), "sm_scale": 1.0 / math.sqrt(d)}
    s["k_pages"] = normal(pool, hkv, PAGE, d)
    s["v_pages"] = normal(pool, hkv, PAGE, d)
    s["q"] = normal(t, hq, d)
    s["out"] = torch.empty_like(s["q"])
    s["context_len"] = _i32(end)
    if kind == "decode":
        s["max_context"] = int(case["len_hi"])
        return s
    s["indptr"], s["indptr_host"], s["context_len_host"] = _i32(indptr), indptr, end.astype(np.int32)
    if kind == "tree":
        s["k_tree"], s["v_tree"] = normal(t, hkv, d), normal(t, hkv, d)
        # trees as beam search drafts them: a node's parent is one of the few before it
        local = torch.arange(t, device=DEVICE) - s["indptr"][:-1].repeat_interleave(_i32(new))
        back = torch.randint(1, 9, (t,), generator=g, device=DEVICE)
        s["parent"] = torch.where(local == 0, -1, (local - back).clamp_min(0)).int()
    return s


def _prepare_pages(case, seed):
    g = np.random.Generator(np.random.PCG64([seed, case["pages"], case["stride"]]))
    kind, n, stride, pages = case["kind"], case["requests"], case["stride"], case["pages"]
    s = {"case": case}

    def deal(have):
        """Every entry where `have` is true gets a page of its own, as far as there are any."""
        most = int(pages * (case["fill"] if kind == "update" else case["used"] if kind == "compact" else 1))
        table = np.full(have.shape, -1)
        at = np.flatnonzero(have)[:most]
        table.reshape(-1)[at] = g.permutation(pages)[:at.size]
        refs = np.zeros(pages, np.int32)
        refs[table[table >= 0]] = 1
        return table, refs

    e = np.arange(stride)[None, :]
    if kind == "update":
        length = g.integers(0, case["len_hi"] + 1, n)
        # what left the window up to `lag` tokens ago is still there
        first = np.maximum(length + 1 - case["window"] - g.integers(0, case["lag"] + 1, n), 0)[:, None]
        kept = (e * PAGE < case["sinks"]) | ((e + 1) * PAGE > first) | (case["window"] == 0)
        table, refs = deal((e * PAGE < length[:, None]) & kept)
        # some pages belong to a prefix that another program keeps
        refs[g.random(pages) < 0.02] += 1
        need = np.minimum(length + g.integers(case["grow_lo"], case["grow_hi"] + 1, n), stride * PAGE)
        over = g.random(n) < case["over"]
        s["context_len"], s["need_len"] = _i32(np.where(over, -1, length)), _i32(need)
        s["capacity"] = torch.empty(n, dtype=torch.int32, device=DEVICE)
    elif kind == "fork":
        length = g.integers(case["len_lo"], case["len_hi"] + 1, case["sources"])
        table, refs = deal(e * PAGE < length[:, None])
        if case["beams"]:
            group = np.arange(n) // case["beams"] * case["beams"]
            source = np.sort(group + g.integers(0, case["beams"], n) * g.integers(0, 2, n))
        else:
            source = g.integers(0, case["sources"], n)
        s["source"], s["context_len"] = _i32(source), _i32(length)
        s["new_context_len"], s["copy_src"], s["copy_dst"] = (torch.empty(n, dtype=torch.int32, device=DEVICE) for _ in range(3))
    else:
        table, refs = deal(g.random((n, stride)) < 0.97)
        s["new_place"], s["move_src"], s["move_dst"] = (torch.empty(pages, dtype=torch.int32, device=DEVICE) for _ in range(3))
        s["counts"] = torch.empty(2, dtype=torch.int32, device=DEVICE)
    s["block_table"], s["page_refs"] = _i32(table), _i32(refs)
    s["new_block_table"] = torch.empty(n, stride, dtype=torch.int32, device=DEVICE)
    s["new_page_refs"] = torch.empty(pages, dtype=torch.int32, device=DEVICE)
    if kind != "update":
        gen = _rng(seed)
        shape = (case["layers"], pages, case["hkv"], PAGE, case["dim"])
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s["k_pages"] = torch.empty(shape, dtype=dtype, device=DEVICE).normal_(generator=gen)
        s["v_pages"] = torch.empty(shape, dtype=dtype, device=DEVICE).normal_(generator=gen)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _gathered(pool, table, place, ok):
    """Keys or values at places [blocks, places] of the rows of `table` [blocks, stride]: [blocks, kv-heads, places, dim]."""
    page = torch.gather(table, 1, torch.where(ok, place // PAGE, 0)).clamp_min(0)
    return pool[page, :, torch.where(ok, place % PAGE, 0)].float().transpose(1, 2)


def _weighted(q, k, v, hidden, scale):
    """q [blocks, kv-heads, rows, dim] over k, v [blocks, kv-heads, keys, dim], but for `hidden` [blocks, rows, keys]."""
    p = (q @ k.transpose(2, 3)) * scale
    p.masked_fill_(hidden[:, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    return (p @ v) / torch.where(total == 0, 1.0, total)


def _prepared(q, pos, first, band, s):
    """q [blocks, rows, heads, dim] at positions pos [blocks, rows] (-1: no row) of the requests whose table rows, lengths and
    first places of the window come with them, the sinks and `band` places from there on gathered, and what each row of q
    does not see: what _weighted takes."""
    c = s["case"]
    n, rows, hq, d = q.shape
    g = hq // c["hkv"]
    table, length = s["table_rows"], s["length_rows"]
    sink = torch.arange(c["sinks"], device=q.device)[None, :].expand(n, -1)
    near = first[:, None] + torch.arange(band, device=q.device)[None, :]
    place = torch.cat([sink, near], 1)
    ok = place < length[:, None]
    ok[:, c["sinks"]:] &= near >= c["sinks"]
    k, v = _gathered(s["k_pages"], table, place, ok), _gathered(s["v_pages"], table, place, ok)
    at = place[:, None, :]
    hidden = ~ok[:, None, :] | (at > pos[:, :, None]) | ((at >= c["sinks"]) & (at <= pos[:, :, None] - c["window"]))
    x = q.float().view(n, rows, c["hkv"], g, d).transpose(1, 2).reshape(n, c["hkv"], rows * g, d)
    return x, k, v, hidden


def _rows_back(o, rows, hq):
    n, hkv, _, d = o.shape
    return o.view(n, hkv, rows, hq // hkv, d).transpose(1, 2).reshape(n, rows, hq, d)


def _prompt_plain(s):
    c = s["case"]
    t, hq, d = s["q"].shape
    new = np.diff(s["indptr_host"])
    blocks = -(-new // BLOCK)
    owner = np.repeat(np.arange(c["requests"]), blocks)
    inside = np.arange(owner.size) - np.repeat(np.cumsum(blocks) - blocks, blocks)
    row0 = _i32(inside * BLOCK).long()
    r = _i32(owner).long()
    indptr = s["indptr"].long()
    row = row0[:, None] + torch.arange(BLOCK, device=DEVICE)[None, :]
    n = (indptr[1:] - indptr[:-1])[r]
    there = row < n[:, None]
    token = torch.where(there, indptr[r][:, None] + row, 0)
    pos = torch.where(there, s["context_len"][r].long()[:, None] - n[:, None] + row, -1)
    longest = int(s["context_len_host"].max())
    band = min(c["window"] - 1 + BLOCK, longest)
    first = (pos[:, 0] - (c["window"] - 1)).clamp_min(0)
    s = {**s, "table_rows": s["block_table"].long()[r], "length_rows": s["context_len"].long()[r]}
    x, k, v, hidden = _prepared(s["q"][token], pos, first, band, s)
    o = _weighted(x, k, v, hidden.repeat_interleave(hq // c["hkv"], 1), s["sm_scale"])
    return _packed(_rows_back(o, BLOCK, hq), token, there, t).to(s["q"].dtype)


def _packed(o, token, there, t):
    """The rows of `o` that are there, at their t tokens (the others go to a row behind them)."""
    whole = torch.empty(t + 1, *o.shape[2:], device=o.device)
    whole[torch.where(there, token, t)] = o
    return whole[:t]


def _decode_plain(s):
    c = s["case"]
    n, hq, d = s["q"].shape
    length = s["context_len"].long()
    band = min(c["window"], s["max_context"])
    s = {**s, "table_rows": s["block_table"].long(), "length_rows": length}
    x, k, v, hidden = _prepared(s["q"][:, None], (length - 1)[:, None], (length - band).clamp_min(0), band, s)
    return _rows_back(_weighted(x, k, v, hidden.expand(-1, hq // c["hkv"], -1), s["sm_scale"]), 1, hq)[:, 0].to(s["q"].dtype)


def _tree_plain(s):
    c = s["case"]
    t, hq, d = s["q"].shape
    n, hkv = c["requests"], c["hkv"]
    g = hq // hkv
    indptr, length = s["indptr"].long(), s["context_len"].long()
    new = indptr[1:] - indptr[:-1]
    most = int(np.diff(s["indptr_host"]).max())
    node = torch.arange(most, device=DEVICE)
    there = node[None, :] < new[:, None]
    token = torch.where(there, indptr[:-1, None] + node, 0)
    parent = torch.where(there & (node > 0), s["parent"].long()[token], -1)
    up = torch.eye(most, device=DEVICE) + (parent[:, :, None] == node).float()
    for _ in range(7):                                  # paths of up to 128 nodes
        up = (up @ up > 0).float()
    depth = up.sum(-1).long() - 1
    pos = torch.where(there, length[:, None] + depth, -1)
    band = min(c["window"] - 1, int(s["context_len_host"].max()))
    s = {**s, "table_rows": s["block_table"].long(), "length_rows": length}
    x, k, v, hidden = _prepared(s["q"][token], pos, (length + 1 - c["window"]).clamp_min(0), band, s)
    own_k, own_v = (s[name][token].float().transpose(1, 2) for name in ("k_tree", "v_tree"))
    near = (pos[:, :, None] - pos[:, None, :] < c["window"]) | (pos[:, None, :] < c["sinks"])
    hidden = torch.cat([hidden, ~((up > 0) & near & there[:, None, :])], 2)
    o = _weighted(x, torch.cat([k, own_k], 2), torch.cat([v, own_v], 2), hidden.repeat_interleave(g, 1), s["sm_scale"])
    return _packed(_rows_back(o, most, hq), token, there, t).to(s["q"].dtype)


def _freed(free):
    """Places of the truths in order, then of the others."""
    return torch.argsort((~free).int(), stable=True)


def _update_plain(s):
    c, table = s["case"], s["block_table"].long()
    pages, stride = s["page_refs"].numel(), table.shape[1]
    length, need = s["context_len"].long()[:, None], s["need_len"].long()[:, None]
    e = torch.arange(stride, device=DEVICE)[None, :]
    has = (table >= 0) & (table < pages)
    over = length < 0
    drop = over.expand_as(table)
    if c["window"]:
        drop = drop | ((e * PAGE >= c["sinks"]) & ((e + 1) * PAGE <= length + 1 - c["window"]))
    refs = s["page_refs"].long().scatter_add(0, table.clamp(0, pages - 1).flatten(), -(drop & has).long().flatten())
    table = torch.where(drop, -1, table)
    has &= ~drop
    last = torch.clamp((need + PAGE - 1) // PAGE, max=stride)
    want = ~over & (e >= (length + PAGE - 1) // PAGE) & (e < last) & ~has
    rank = (torch.cumsum(want.flatten().long(), 0) - 1).view_as(table)
    free = refs <= 0
    got = want & (rank < free.sum())
    table = torch.where(got, _freed(free)[rank.clamp(0, pages - 1)], table)
    refs = torch.where(free & (torch.cumsum(free.long(), 0) <= got.sum()), 1, refs)
    without = (need > length) & (e >= length // PAGE) & (e < last) & ~has & ~got
    reach = torch.where(without, torch.maximum(e * PAGE, length), torch.clamp(need, max=stride * PAGE)).amin(1)
    return {"block_table": table.int(), "page_refs": refs.int(), "capacity": torch.where(over[:, 0], 0, reach).int()}


def _copied(s, src, dst):
    """Pages src to pages dst (-1: nothing, which repeats the first copy, or page 0 to itself) of all layers."""
    real = dst >= 0
    one = real.int().argmax()
    src, dst = (torch.where(real, x, torch.where(real[one], x[one], 0)) for x in (src, dst))
    for name in ("k_pages", "v_pages"):
        s[name][:, dst] = s[name][:, src]


def _fork_plain(s):
    table = s["block_table"].long()
    sources, stride = table.shape
    pages, n = s["page_refs"].numel(), s["source"].numel()
    source = s["source"].long()
    ok = (source >= 0) & (source < sources)
    source = source.clamp(0, sources - 1)
    length = s["context_len"].long().clamp(0, stride * PAGE)
    whole = length // PAGE
    takers = torch.zeros(sources, dtype=torch.long, device=DEVICE).scatter_add(0, source, ok.long())
    row = torch.arange(n, device=DEVICE)
    first = torch.full((sources,), n, device=DEVICE).scatter_reduce(0, source, torch.where(ok, row, n), "amin")
    is_first = ok & (first[source] == row)
    e = torch.arange(stride, device=DEVICE)[None, :]
    has = (table >= 0) & (table < pages)
    more = torch.where(e < whole[:, None], takers[:, None] - 1, torch.where(takers > 0, 0, -1)[:, None])
    refs = s["page_refs"].long().scatter_add(0, table.clamp(0, pages - 1).flatten(), (more * has).flatten())
    at = whole[source]
    taken = ok[:, None] & ((e < at[:, None]) | is_first[:, None])
    new = torch.where(taken, table[source], -1)
    inside = at.clamp(max=stride - 1)
    old = table[source, inside]
    want = ok & ~is_first & (length[source] % PAGE != 0) & has[source, inside]
    rank = torch.cumsum(want.long(), 0) - 1
    free = refs <= 0
    got = want & (rank < free.sum())
    page = _freed(free)[rank.clamp(0, pages - 1)]
    new = torch.where(got[:, None] & (e == at[:, None]), page[:, None], new)
    refs = torch.where(free & (torch.cumsum(free.long(), 0) <= got.sum()), 1, refs)
    src, dst = torch.where(got, old, -1), torch.where(got, page, -1)
    _copied(s, src, dst)
    length = torch.where(ok, torch.where(want & ~got, at * PAGE, length[source]), 0)
    return {"block_table": new.int(), "page_refs": refs.int(), "context_len": length.int(), "src": src.int(), "dst": dst.int(),
            "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _compact_plain(s):
    refs, table = s["page_refs"].long(), s["block_table"].long()
    pages = refs.numel()
    used = refs > 0
    count = used.sum()
    p = torch.arange(pages, device=DEVICE)
    mover, hole = used & (p >= count), ~used & (p < count)
    moves = mover.sum()
    src, dst = torch.where(p < moves, _freed(mover), -1), torch.where(p < moves, _freed(hole), -1)
    rank = (torch.cumsum(mover.long(), 0) - 1).clamp_min(0)
    place = torch.where(mover, dst[rank], torch.where(used, p, -1))
    moved = torch.zeros(pages + 1, dtype=torch.long, device=DEVICE).scatter(0, torch.where(used, place, pages), refs)[:pages]
    has = (table >= 0) & (table < pages)
    most = max(1, pages // 2)                           # (as many holes at least as moves)
    _copied(s, src[:most], dst[:most])
    return {"block_table": torch.where(has, place[table.clamp(0, pages - 1)], table).int(), "page_refs": moved.int(),
            "place": place.int(), "src": src.int(), "dst": dst.int(), "counts": torch.stack([count, moves]).int(),
            "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _workspace(s, query):
    """Made on a state's first pass and kept, as a program keeps it beside its cache."""
    if "workspace" not in s:
        need = query()
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEVICE) if need else None
    return s["workspace"]


def _own(s):
    import paper_2501_12162_amd as ada
    c = s["case"]
    kind = c["kind"]
    if kind in ("update", "fork", "compact"):
        return _own_pages(ada, s)
    code = ada.ADASERVE_BF16 if c["dtype"] == "bf16" else ada.ADASERVE_F32
    shape = (c["hq"], c["hkv"], c["dim"], PAGE, c["window"], c["sinks"], code)
    cache = {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "block_table": s["block_table"], "window": c["window"],
             "sinks": c["sinks"], "sm_scale": s["sm_scale"], "q": s["q"], "out": s["out"]}
    if kind == "decode":
        ws = _workspace(s, lambda: ada.adaserve_window_decode_attn_workspace_bytes(c["requests"], s["max_context"], *shape))
        ada.adaserve_window_decode_attn(context_len=s["context_len"], max_context=min(s["max_context"], s["block_table"].shape[1] * PAGE),
                                        workspace=ws, **cache)
    elif kind == "prompt":
        ws = _workspace(s, lambda: ada.adaserve_window_prompt_attn_workspace_bytes(s["indptr_host"], s["context_len_host"], *shape))
        ada.adaserve_window_prompt_attn(token_indptr=s["indptr"], token_indptr_host=s["indptr_host"], context_len=s["context_len"],
                                        context_len_host=s["context_len_host"], workspace=ws, **cache)
    else:
        ws = _workspace(s, lambda: ada.adaserve_window_tree_attn_workspace_bytes(s["indptr_host"], s["context_len_host"], *shape))
        ada.adaserve_window_tree_attn(node_indptr=s["indptr"], node_indptr_host=s["indptr_host"], parent=s["parent"],
                                      k_tree=s["k_tree"], v_tree=s["v_tree"], prefix_len=s["context_len"],
                                      prefix_len_host=s["context_len_host"], workspace=ws, **cache)
    return s["out"]


def _own_pages(ada, s):
    c = s["case"]
    rows = max(c["requests"], c.get("sources", 0))
    ws = _workspace(s, lambda: ada.adaserve_pages_workspace_bytes(rows, c["pages"]))
    tables = {"block_table": s["block_table"], "page_refs": s["page_refs"], "new_block_table": s["new_block_table"],
              "new_page_refs": s["new_page_refs"], "workspace": ws}
    out = {"block_table": s["new_block_table"], "page_refs": s["new_page_refs"]}
    if c["kind"] == "update":
        ada.adaserve_update_pages(context_len=s["context_len"], need_len=s["need_len"], window=c["window"], sinks=c["sinks"],
                                  page_size=PAGE, capacity=s["capacity"], **tables)
        return {**out, "capacity": s["capacity"]}
    if c["kind"] == "fork":
        ada.adaserve_fork_pages(source=s["source"], context_len=s["context_len"], page_size=PAGE,
                                new_context_len=s["new_context_len"], copy_src=s["copy_src"], copy_dst=s["copy_dst"], **tables)
        ada.adaserve_copy_pages(src=s["copy_src"], dst=s["copy_dst"], k_pages=s["k_pages"], v_pages=s["v_pages"])
        return {**out, "context_len": s["new_context_len"], "src": s["copy_src"], "dst": s["copy_dst"], "k_pages": s["k_pages"],
                "v_pages": s["v_pages"]}
    ada.adaserve_compact_pages(new_place=s["new_place"], move_src=s["move_src"], move_dst=s["move_dst"], counts=s["counts"], **tables)
    ada.adaserve_copy_pages(src=s["move_src"], dst=s["move_dst"], count=s["counts"][1:], k_pages=s["k_pages"], v_pages=s["v_pages"])
    return {**out, "place": s["new_place"], "src": s["move_src"], "dst": s["move_dst"], "counts": s["counts"],
            "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def run(state):
    if own:
        return _own(state)
    return {"prompt": _prompt_plain, "decode": _decode_plain, "tree": _tree_plain, "update": _update_plain,
            "fork": _fork_plain, "compact": _compact_plain}[state["case"]["kind"]](state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("update", "fork", "compact"):
        return {"update": _update_exact, "fork": _fork_exact, "compact": _compact_exact}[case["kind"]](s)
    before, new = _lens(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    hkv, g, row = case["hkv"], case["hq"] // case["hkv"], 0
    for r, (b, n) in enumerate(zip(before.tolist(), new.tolist())):
        ctx = b + n if case["kind"] == "prompt" else b
        place = torch.arange(ctx, device=DEVICE)
        page = s["block_table"][r].long()[place // PAGE].clamp_min(0)
        if case["kind"] == "tree":
            parent = s["parent"][row:row + n].tolist()
            paths = []
            for i in range(n):
                paths.append(([] if i == 0 else paths[parent[i]]) + [i])
            pos = torch.tensor([b + len(p) - 1 for p in paths], device=DEVICE)
            on = torch.zeros(n, n, dtype=torch.bool)
            for i, p in enumerate(paths):
                on[i, p] = True
            at = torch.cat([place, pos])
            seen = torch.cat([torch.ones(n, b, dtype=torch.bool, device=DEVICE), on.to(DEVICE)], 1)
        else:
            pos = torch.arange(ctx - n, ctx, device=DEVICE)
            at = place
            seen = place[None, :] <= pos[:, None]
        seen = seen & ((at[None, :] > pos[:, None] - case["window"]) | (at[None, :] < case["sinks"]))
        if n and at.numel() and seen.any():
            none = ~seen.any(1)
            for h in range(hkv):
                k = s["k_pages"][page, h, place % PAGE].double()
                v = s["v_pages"][page, h, place % PAGE].double()
                if case["kind"] == "tree":
                    k = torch.cat([k, s["k_tree"][row:row + n, h].double()])
                    v = torch.cat([v, s["v_tree"][row:row + n, h].double()])
                for x in range(h * g, (h + 1) * g):
                    z = s["q"][row:row + n, x].double() @ k.T * s["sm_scale"]
                    p = torch.softmax(z.masked_fill_(~seen, -math.inf), 1)
                    out[row:row + n, x] = torch.where(none[:, None], 0.0, p) @ v
        row += n
    return out


def _lists(s, *names):
    return [s[name].cpu().tolist() for name in names]


def _update_exact(s):
    c = s["case"]
    table, refs, length, need = _lists(s, "block_table", "page_refs", "context_len", "need_len")
    for r, row in enumerate(table):
        for e, p in enumerate(row):
            gone = length[r] < 0
            if c["window"] and not gone:
                gone = all(j >= c["sinks"] and j <= length[r] - c["window"] for j in range(e * PAGE, (e + 1) * PAGE, PAGE - 1))
            if gone:
                row[e] = -1
                if 0 <= p < len(refs):
                    refs[p] -= 1
    free = iter([p for p, n in enumerate(refs) if n <= 0])
    capacity = []
    for r, row in enumerate(table):
        if length[r] < 0:
            capacity.append(0)
            continue
        for e in range(-(-length[r] // PAGE), min(-(-need[r] // PAGE), len(row))):
            if not 0 <= row[e] < len(refs):
                p = next(free, None)
                if p is None:
                    break
                row[e], refs[p] = p, 1
        at, limit = length[r], min(need[r], len(row) * PAGE)
        while at < limit and 0 <= row[at // PAGE] < len(refs):
            at = at // PAGE * PAGE + PAGE
        capacity.append(min(at, limit))
    return {"block_table": _i32(table), "page_refs": _i32(refs), "capacity": _i32(capacity)}


def _fork_exact(s):
    table, refs, length, source = _lists(s, "block_table", "page_refs", "context_len", "source")
    stride = len(table[0])
    length = [min(max(x, 0), stride * PAGE) for x in length]
    inside = lambda p: 0 <= p < len(refs)  # noqa: E731
    seen, new, kept = set(), [], []
    for r, f in enumerate(source):
        if not 0 <= f < len(table):
            new.append([-1] * stride)
            kept.append(0)
            continue
        n = length[f] // PAGE
        new.append(table[f][:] if f not in seen else table[f][:n] + [-1] * (stride - n))
        kept.append(length[f])
        for p in table[f][:n] if f in seen else table[f]:
            if inside(p):
                refs[p] += 1
        seen.add(f)
    for row in table:
        for p in row:
            if inside(p):
                refs[p] -= 1
    free = iter([p for p, n in enumerate(refs) if n <= 0])
    src, dst, seen = [-1] * len(source), [-1] * len(source), set()
    for r, f in enumerate(source):
        if 0 <= f < len(table):
            n = length[f] // PAGE
            if f in seen and length[f] % PAGE and inside(table[f][n]):
                p = next(free, None)
                if p is None:
                    kept[r] = n * PAGE
                else:
                    src[r], dst[r], new[r][n], refs[p] = table[f][n], p, p, 1
            seen.add(f)
    pools = [s[name].clone() for name in ("k_pages", "v_pages")]
    for pool in pools:
        for a, b in zip(src, dst):
            if b >= 0:
                pool[:, b] = pool[:, a]
    return {"block_table": _i32(new), "page_refs": _i32(refs), "context_len": _i32(kept), "src": _i32(src), "dst": _i32(dst),
            "k_pages": pools[0].double(), "v_pages": pools[1].double()}


def _compact_exact(s):
    table, refs = _lists(s, "block_table", "page_refs")
    used = [p for p, n in enumerate(refs) if n > 0]
    holes = [p for p, n in enumerate(refs) if n <= 0 and p < len(used)]
    movers = [p for p in used if p >= len(used)]
    place = [p if n > 0 else -1 for p, n in enumerate(refs)]
    for a, b in zip(movers, holes):
        place[a] = b
    moved = [0] * len(refs)
    for p in used:
        moved[place[p]] = refs[p]
    table = [[place[p] if 0 <= p < len(refs) else p for p in row] for row in table]
    rest = [-1] * (len(refs) - len(movers))
    pools = [s[name].clone() for name in ("k_pages", "v_pages")]
    if movers:
        a, b = torch.tensor(movers, device=DEVICE), torch.tensor(holes, device=DEVICE)
        for pool in pools:
            pool[:, b] = pool[:, a]
    return {"block_table": _i32(table), "page_refs": _i32(moved), "place": _i32(place), "src": _i32(movers + rest),
            "dst": _i32(holes + rest), "counts": _i32([len(used), len(movers)]), "k_pages": pools[0].double(),
            "v_pages": pools[1].double()}
