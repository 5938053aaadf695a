"""The serving operators around tree verification, with inputs as a serving program has them.

A case is one call:

* ``append``  rotary position embedding of queries and keys, and the keys and values written into the paged cache
              (a prompt's tokens, one token of every request, or the nodes of draft trees, which are rotated only);
* ``prompt``  causal attention of the tokens of packed prompts, or of a chunk of each, over the paged cache;
* ``decode``  attention of one new token per request over the paged cache;
* ``sample``  a token per row of logits by temperature, top-k, top-p and min-p, from given random numbers.

Lengths come from the case (``sizes`` seeds them), values and page places from ``prepare``'s seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
PAGE = 16
UNIT = 4294967296.0   # a token's mass is held in whole units of 2^-32 of the likeliest token's

# The dearest drawn case stays within these (one pass of the largest listed ones).
MOST_PROMPT_FLOPS = 5.5e11
MOST_PROMPT_FLOPS_F32 = 1.5e10
MOST_SCORES = 2.4e9          # padded scores of the plain form
MOST_CACHE_BYTES = 1.07e9
MOST_TOKENS = 13000
MOST_LOGIT_BYTES = 1.31e8


def listed():
    chat = {"hq": 32, "hkv": 8, "dim": 128, "dtype": "bf16"}
    big = {"hq": 64, "hkv": 8, "dim": 128, "dtype": "bf16"}
    return [
        # The smallest call: the one new token of an idle server's only user.
        {"name": "append_one_user", "kind": "append", "requests": 1, "new_lo": 1, "new_hi": 1, "len_lo": 1500,
         "len_hi": 1500, "rotary": 128, "interleaved": False, "tree": False, "sizes": 1, **chat},
        # The prompts of eight chat requests as they arrive, ragged.
        {"name": "append_8b_prompts", "kind": "append", "requests": 8, "new_lo": 300, "new_hi": 2500, "len_lo": 0,
         "len_hi": 0, "rotary": 128, "interleaved": False, "tree": False, "sizes": 2, **chat},
        # Draft trees of 16 requests before their verification in fp32: nodes at their depths, half of each head rotated in
        # neighbouring pairs, nothing appended.
        {"name": "append_tree_f32", "kind": "append", "requests": 16, "new_lo": 8, "new_hi": 64, "len_lo": 512,
         "len_hi": 2048, "hq": 16, "hkv": 4, "dim": 128, "dtype": "f32", "rotary": 64, "interleaved": True, "tree": True,
         "sizes": 3},
        # Attention over 16 chat prompts at once, ragged: the usual prefill of one layer.
        {"name": "prompt_8b", "kind": "prompt", "requests": 16, "new_lo": 512, "new_hi": 2048, "len_lo": 0, "len_hi": 0,
         "sizes": 4, **chat},
        # One long document: the largest matrix work.
        {"name": "prompt_long", "kind": "prompt", "requests": 1, "new_lo": 8191, "new_hi": 8191, "len_lo": 0, "len_hi": 0,
         "sizes": 5, **chat},
        # Chunked prefill beside decoding: small chunks of four long prompts over what is cached of them already.
        {"name": "prompt_chunks_70b", "kind": "prompt", "requests": 4, "new_lo": 64, "new_hi": 256, "len_lo": 4096,
         "len_hi": 8192, "sizes": 6, **big},
        # fp32 prompts of a small batch with head dimension 64, as a numerics run of a model makes it.
        {"name": "prompt_f32", "kind": "prompt", "requests": 3, "new_lo": 1, "new_hi": 700, "len_lo": 0, "len_hi": 100,
         "hq": 8, "hkv": 8, "dim": 64, "dtype": "f32", "sizes": 7},
        # The next token of an idle server's only user: latency.
        {"name": "decode_one_user", "kind": "decode", "requests": 1, "len_lo": 1500, "len_hi": 1500, "sizes": 8, **chat},
        # Every request of a full server with the 70B shape's heads, ragged, some of them padding of the batch (length 0).
        {"name": "decode_70b", "kind": "decode", "requests": 64, "len_lo": 0, "len_hi": 4096, "sizes": 9, **big},
        # Long documents: 32768 cached tokens each, the largest cache traffic.
        {"name": "decode_long_context", "kind": "decode", "requests": 8, "len_lo": 32768, "len_hi": 32768, "sizes": 10,
         **chat},
        # One user's next token.
        {"name": "sample_one_user", "kind": "sample", "requests": 1, "vocab": 128256, "pad": 0, "dtype": "bf16", "spread": 2.0,
         "mix": "chat"},
        # A full server's next tokens, every row with parameters of its own.
        {"name": "sample_batch_f32", "kind": "sample", "requests": 250, "vocab": 128256, "pad": 8, "dtype": "f32",
         "spread": 2.0, "mix": "all"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choices(["append", "prompt", "decode", "sample"], [2, 3, 3, 3])[0]
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    c = {"kind": kind, "dtype": dtype, "sizes": rng.randrange(1 << 20)}
    if kind == "sample":
        c["vocab"] = rng.choice([128256, 151936, 32064, 50257, _log_int(rng, 100, 128000)])
        c["pad"] = rng.choice([0, 0, 1, 8, 64])
        c["requests"] = _log_int(rng, 1, max(1, min(512, int(MOST_LOGIT_BYTES / (_size(c) * (c["vocab"] + c["pad"]))))))
        c["spread"] = rng.choice([0.5, 1.0, 2.0, 4.0, 8.0])
        c["mix"] = rng.choice(["all", "all", "chat", "free"])
        return c
    c["hq"], c["hkv"] = rng.choice([(32, 8), (64, 8), (16, 2), (8, 8), (16, 4), (32, 2), (16, 16), (4, 2), (28, 4), (6, 2)])
    c["dim"] = 128 if rng.random() < 0.75 else 64
    c["requests"] = _log_int(rng, 1, 64)
    if kind == "append":
        c["tree"] = rng.random() < 0.25
        c["new_hi"] = 1 if rng.random() < 0.4 else _log_int(rng, 1, 128 if c["tree"] else 4096)
        c["new_lo"] = 1 if c["new_hi"] == 1 else rng.randint(0, c["new_hi"])
        c["requests"] = max(1, min(c["requests"], MOST_TOKENS // c["new_hi"]))
        c["len_hi"] = rng.choice([0, _log_int(rng, 1, 32768)])
        c["len_lo"] = rng.randint(0, c["len_hi"])
        c["new_lo"] = max(c["new_lo"], int(_lens(c)[1].sum() == 0))
        c["rotary"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2])
        c["interleaved"] = rng.random() < 0.3
        return c
    if kind == "decode":
        c["len_hi"] = _log_int(rng, 1, 32768)
        c["len_lo"] = rng.randint(0, c["len_hi"])
        while c["requests"] > 1 and c["requests"] * c["len_hi"] * c["hkv"] * c["dim"] * 2 * _size(c) > MOST_CACHE_BYTES:
            c["requests"] = c["requests"] * 3 // 4
        c["len_lo"] = max(c["len_lo"], int(_lens(c)[0].sum() == 0))
        return c
    c["new_hi"] = _log_int(rng, 1, 8192)
    c["new_lo"] = rng.randint(0, c["new_hi"])
    c["len_hi"] = rng.choice([0, _log_int(rng, 1, 8192)])
    c["len_lo"] = rng.randint(0, c["len_hi"])
    most = MOST_PROMPT_FLOPS if dtype == "bf16" else MOST_PROMPT_FLOPS_F32
    while True:
        scores = c["requests"] * c["hq"] * c["new_hi"] * (c["new_hi"] + c["len_hi"] + 16.0)
        if scores <= MOST_SCORES and work(c)["flops"] <= most:
            c["new_lo"] = max(c["new_lo"], int(_lens(c)[1].sum() == 0))
            return c
        if c["requests"] > 1 and (rng.random() < 0.6 or c["new_hi"] < 64):
            c["requests"] = c["requests"] * 3 // 4
        elif c["new_hi"] >= 64:
            c["new_hi"] = c["new_hi"] * 3 // 4
            c["new_lo"] = min(c["new_lo"], c["new_hi"])
        else:
            c["len_hi"] = c["len_hi"] * 3 // 4
            c["len_lo"] = min(c["len_lo"], c["len_hi"])


def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _lens(case):
    """Cached tokens before the call and new tokens, per request."""
    g = np.random.Generator(np.random.PCG64(case["sizes"]))
    before = g.integers(case["len_lo"], case["len_hi"] + 1, case["requests"])
    if case["kind"] == "decode":
        return before, np.ones_like(before)
    new = g.integers(case["new_lo"], case["new_hi"] + 1, case["requests"])
    return before, new


def work(case):
    s = _size(case)
    n = case["requests"]
    if case["kind"] == "sample":
        return {"bytes": n * (case["vocab"] * s + 4 * 6), "flops": n * case["vocab"] * 8}
    before, new = (a.astype(np.float64) for a in _lens(case))
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    if case["kind"] == "append":
        t = float(new.sum())
        moved = 2 * (hq + hkv) + (0 if case["tree"] else 2 * hkv)   # q, k (and v), each read and written
        return {"bytes": t * moved * d * s + 8 * n + 2 * case["rotary"], "flops": t * (hq + hkv) * case["rotary"] * 3}
    if case["kind"] == "decode":
        keys = float(before.sum())
        return {"bytes": 2 * keys * hkv * d * s + 2 * n * hq * d * s + keys / PAGE * 4, "flops": 4 * keys * hq * d}
    seen = float((new * before + new * (new + 1) / 2).sum())
    ctx = float((before + new)[new > 0].sum())
    return {"bytes": 2 * ctx * hkv * d * s + 2 * float(new.sum()) * hq * d * s, "flops": 4 * seen * hq * d}


def _rng(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device=DEVICE)


def prepare(case, seed):
    g = _rng(seed)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    n = case["requests"]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device=DEVICE) * std).to(dtype)

    def uniform(lo, hi):
        return torch.rand(n, generator=g, device=DEVICE) * (hi - lo) + lo

    if case["kind"] == "sample":
        v = case["vocab"]
        logits = torch.randn(n, v + case["pad"], generator=g, device=DEVICE) * case["spread"]
        # a few likely tokens stand out of the bulk, as after most contexts
        likely = torch.randint(v, (n, 24), generator=g, device=DEVICE)
        logits.scatter_add_(1, likely, torch.rand(n, 24, generator=g, device=DEVICE) * 5 * case["spread"])
        s = {"case": case, "logits": logits.to(dtype), "u": torch.rand(n, generator=g, device=DEVICE)}
        row = torch.arange(n, device=DEVICE)
        s["temperature"] = uniform(0.5, 1.3)
        s["top_k"] = torch.randint(1, 101, (n,), generator=g, device=DEVICE).int()
        s["top_p"] = uniform(0.5, 1.0)
        s["min_p"] = uniform(0.0, 0.1)
        if case["mix"] == "chat":       # what most chat servers set
            s["temperature"].fill_(0.7)
            s["top_k"].fill_(50)
            s["top_p"].fill_(0.9)
            s["min_p"].zero_()
        elif case["mix"] == "free":     # the whole distribution
            s["temperature"].fill_(1.0)
            s["top_k"].zero_()
            s["top_p"].fill_(1.0)
            s["min_p"].zero_()
        else:                           # users differ: greedy ones, ones without one filter or another
            s["temperature"][row % 9 == 4] = 0.0
            s["top_k"][row % 3 != 0] = 0
            s["top_p"][row % 4 == 1] = 1.0
            s["min_p"][row % 2 == 0] = 0.0
        return s

    before, new = _lens(case)
    hq, hkv, d = case["hq"], case["hkv"], case["dim"]
    end = before + new if case["kind"] != "decode" else before
    pages = -(-end // PAGE)
    total = int(pages.sum())
    pool = total + 4
    wide = max(1, int(pages.max()))
    perm = torch.randperm(pool, generator=g, device=DEVICE).cpu().numpy()
    at = (np.cumsum(pages) - pages)[:, None] + np.arange(wide)[None, :]
    table = np.where(np.arange(wide)[None, :] < pages[:, None], perm[np.minimum(at, pool - 1)], -1)
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    t = int(indptr[-1])
    s = {"case": case, "block_table": _i32(table)}
    s["k_pages"] = normal(pool, hkv, PAGE, d)
    s["v_pages"] = normal(pool, hkv, PAGE, d)
    if case["kind"] == "append":
        # the queries, keys and values of a layer lie side by side in the rows of one projection's output
        rows = normal(t, (hq + 2 * hkv) * d)
        s["q"] = rows[:, :hq * d].view(t, hq, d)
        s["k"] = rows[:, hq * d:(hq + hkv) * d].view(t, hkv, d)
        s["v"] = rows[:, (hq + hkv) * d:].view(t, hkv, d)
        s["token_indptr"], s["prefix_len"] = _i32(indptr), _i32(before)
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, case["rotary"], 2, device=DEVICE, dtype=torch.float64) / case["rotary"])).float()
        s["q_out"] = torch.empty(t, hq, d, dtype=dtype, device=DEVICE)
        s["new_prefix_len"] = torch.empty(n, dtype=torch.int32, device=DEVICE)
        s["positions"] = s["k_out"] = None
        if case["tree"]:
            local = np.arange(t) - np.repeat(indptr[:-1], new)
            s["positions"] = _i32(np.repeat(before, new) + np.floor(np.log2(local + 1)))   # two children each
            s["k_out"] = torch.empty(t, hkv, d, dtype=dtype, device=DEVICE)
        return s
    s["sm_scale"] = 1.0 / math.sqrt(d)
    s["context_len"] = _i32(end)
    s["q"] = normal(t, hq, d)
    s["out"] = torch.empty_like(s["q"])
    if case["kind"] == "decode":
        s["max_context"] = int(case["len_hi"])
    else:
        s["token_indptr"], s["token_indptr_host"], s["context_len_host"] = _i32(indptr), indptr, end.astype(np.int32)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _rows(indptr, t):
    """Request and place in it of each of t tokens."""
    token = torch.arange(t, device=indptr.device)
    r = torch.searchsorted(indptr, token.to(indptr.dtype), right=True) - 1
    return r, token - indptr[r]


def _rotated(x, angle, rotary, interleaved):
    x = x.float()
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rotary:2], x[..., 1:rotary:2]
        y[..., 0:rotary:2], y[..., 1:rotary:2] = a * cos - b * sin, a * sin + b * cos
    else:
        h = rotary // 2
        a, b = x[..., :h], x[..., h:rotary]
        y[..., :h], y[..., h:rotary] = a * cos - b * sin, a * sin + b * cos
    return y


def _append_plain(s):
    c = s["case"]
    r, i = _rows(s["token_indptr"], s["q"].shape[0])
    place = s["prefix_len"][r] + i
    pos = place if s["positions"] is None else s["positions"]
    angle = pos.double()[:, None] * s["inv_freq"].double()[None, :]
    q = _rotated(s["q"], angle, c["rotary"], c["interleaved"]).to(s["q"].dtype)
    k = _rotated(s["k"], angle, c["rotary"], c["interleaved"]).to(s["k"].dtype)
    if c["tree"]:
        return {"q": q, "k": k}
    page, slot = s["block_table"][r, place // PAGE], place % PAGE
    s["k_pages"][page, :, slot] = k
    s["v_pages"][page, :, slot] = s["v"]
    return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"],
            "new_prefix_len": s["prefix_len"] + s["token_indptr"][1:] - s["token_indptr"][:-1]}


def _cached(pool, table):
    """The requests' pages one after another: [requests, kv-heads, places, dim]."""
    x = pool[table.clamp_min(0)].float()
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _attend(q, pos, s):
    """q [requests, kv-heads, rows, dim] at positions pos [requests, rows] over the cached keys up to them."""
    k, v = _cached(s["k_pages"], s["block_table"]), _cached(s["v_pages"], s["block_table"])
    key = torch.arange(k.shape[2], device=q.device)
    hidden = (key[None, None, :] > pos[:, :, None])[:, None]
    p = (q @ k.transpose(2, 3)) * s["sm_scale"]
    p.masked_fill_(hidden, -math.inf)
    m = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    return (p @ v) / torch.where(total == 0, 1.0, total)


def _prompt_plain(s):
    c = s["case"]
    t, hq, d = s["q"].shape
    n, g = c["requests"], hq // c["hkv"]
    most = int(np.diff(s["token_indptr_host"]).max())
    r, i = _rows(s["token_indptr"], t)
    q = torch.zeros(n, most, hq, d, device=DEVICE)
    q[r, i] = s["q"].float()
    new = s["token_indptr"][1:] - s["token_indptr"][:-1]
    pos = (s["context_len"] - new)[:, None] + torch.arange(most, device=DEVICE)[None, :]
    q = q.view(n, most, c["hkv"], g, d).transpose(1, 2).reshape(n, c["hkv"], most * g, d)
    o = _attend(q, pos.repeat_interleave(g, 1), s)
    o = o.view(n, c["hkv"], most, g, d).transpose(1, 2).reshape(n, most, hq, d)
    return o[r, i].to(s["q"].dtype)


def _decode_plain(s):
    c = s["case"]
    n, hq, d = s["q"].shape
    q = s["q"].float().view(n, c["hkv"], hq // c["hkv"], d)
    pos = (s["context_len"] - 1)[:, None].expand(n, hq // c["hkv"])
    return _attend(q, pos, s).view(n, hq, d).to(s["q"].dtype)


def _sample_plain(s):
    v = s["case"]["vocab"]
    x, index = torch.sort(s["logits"][:, :v].float(), descending=True, stable=True)   # ties: the lowest index first
    z = x.double() - x[:, :1].double()
    t = s["temperature"].double()[:, None]
    w = torch.where(t > 0, torch.round(torch.exp(z / torch.where(t > 0, t, 1.0)) * UNIT), 0.0)
    w[:, 0] = UNIT
    rank = torch.arange(v, device=x.device)[None, :]
    k = s["top_k"].long()[:, None]
    w = torch.where((rank < k) | (k <= 0), w, 0.0)
    before = torch.cumsum(w, 1) - w                   # whole numbers below 2^53: exact in any order
    p = s["top_p"].double()[:, None]
    kept = (before < p * w.sum(1, keepdim=True)) | (p >= 1)
    kept &= w >= s["min_p"].double()[:, None] * UNIT
    kept[:, 0] = True
    mass = torch.zeros_like(w).scatter_(1, index, torch.where(kept, w, 0.0))
    upto = torch.cumsum(mass, 1)
    return (upto <= s["u"].double()[:, None] * upto[:, -1:]).sum(1).int()


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
    code = ada.ADASERVE_BF16 if c["dtype"] == "bf16" else ada.ADASERVE_F32
    if c["kind"] == "append":
        tree = c["tree"]
        ada.adaserve_rope_append_kv(
            token_indptr=s["token_indptr"], prefix_len=s["prefix_len"], positions=s["positions"], q=s["q"], k=s["k"],
            v=None if tree else s["v"], inv_freq=s["inv_freq"], interleaved=c["interleaved"], q_out=s["q_out"],
            k_out=s["k_out"], k_pages=None if tree else s["k_pages"], v_pages=None if tree else s["v_pages"],
            block_table=None if tree else s["block_table"], new_prefix_len=None if tree else s["new_prefix_len"])
        if tree:
            return {"q": s["q_out"], "k": s["k_out"]}
        return {"q": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"], "new_prefix_len": s["new_prefix_len"]}
    if c["kind"] == "prompt":
        ws = _workspace(s, lambda: ada.adaserve_prompt_attn_workspace_bytes(
            s["token_indptr_host"], s["context_len_host"], c["hq"], c["hkv"], c["dim"], PAGE, code))
        ada.adaserve_prompt_attn(
            token_indptr=s["token_indptr"], token_indptr_host=s["token_indptr_host"], q=s["q"], k_pages=s["k_pages"],
            v_pages=s["v_pages"], block_table=s["block_table"], context_len=s["context_len"],
            context_len_host=s["context_len_host"], sm_scale=s["sm_scale"], out=s["out"], workspace=ws)
        return s["out"]
    if c["kind"] == "decode":
        most = min(s["max_context"], s["block_table"].shape[1] * PAGE)   # the bound is at most what the table holds
        ws = _workspace(s, lambda: ada.adaserve_decode_attn_workspace_bytes(
            c["requests"], most, c["hq"], c["hkv"], c["dim"], PAGE, code))
        ada.adaserve_decode_attn(
            q=s["q"], k_pages=s["k_pages"], v_pages=s["v_pages"], block_table=s["block_table"],
            context_len=s["context_len"], max_context=most, sm_scale=s["sm_scale"], out=s["out"], workspace=ws)
        return s["out"]
    if "token" not in s:
        s["token"] = torch.empty(c["requests"], dtype=torch.int32, device=DEVICE)
    ws = _workspace(s, lambda: ada.adaserve_sample_workspace_bytes(c["requests"], c["vocab"], code))
    ada.adaserve_sample(logits=s["logits"], vocab=c["vocab"], temperature=s["temperature"], top_k=s["top_k"],
                        top_p=s["top_p"], min_p=s["min_p"], u=s["u"], out_token=s["token"], workspace=ws)
    return s["token"]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "append":
        return _append_plain(state)
    if kind == "prompt":
        return _prompt_plain(state)
    return _decode_plain(state) if kind == "decode" else _sample_plain(state)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return _sample_exact(s)
    if case["kind"] == "append":
        return _append_exact(s)
    before, new = _lens(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    hkv, g, row = case["hkv"], case["hq"] // case["hkv"], 0
    for r, (b, n) in enumerate(zip(before.tolist(), new.tolist())):
        ctx = b + n if case["kind"] == "prompt" else b
        if n and ctx:
            place = torch.arange(ctx, device=DEVICE)
            page = s["block_table"][r].long()[place // PAGE]
            for h in range(hkv):
                k = s["k_pages"][page, h, place % PAGE].double()
                v = s["v_pages"][page, h, place % PAGE].double()
                for e in range(g):
                    q = s["q"][row:row + n, h * g + e].double()
                    z = q @ k.T * s["sm_scale"]
                    z[place[None, :] > torch.arange(ctx - n, ctx, device=DEVICE)[:, None]] = -math.inf
                    out[row:row + n, h * g + e] = torch.softmax(z, 1) @ v
        row += n
    return out


def _append_exact(s):
    """Pairs as complex numbers turned by e^(i p f)."""
    c, q = s["case"], s["q"].double()
    before, new = _lens(c)
    place = np.concatenate([np.arange(b, b + n) for b, n in zip(before.tolist(), new.tolist())] or [np.zeros(0, int)])
    pos = place if s["positions"] is None else s["positions"].cpu().numpy()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE),
                       torch.outer(torch.as_tensor(pos, device=DEVICE).double(), s["inv_freq"].double()))

    def turned(x):
        x, rot, rest = x.double(), c["rotary"], x.double()[..., c["rotary"]:]
        pair = x[..., :rot].unflatten(-1, (rot // 2, 2) if c["interleaved"] else (2, rot // 2))
        pair = pair if c["interleaved"] else pair.transpose(-1, -2)
        y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None])
        y = y if c["interleaved"] else y.transpose(-1, -2)
        return torch.cat([y.flatten(-2), rest], -1)

    q, k = turned(q), turned(s["k"])
    if c["tree"]:
        return {"q": q, "k": k}
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    table = s["block_table"].cpu().numpy()
    owner = np.repeat(np.arange(c["requests"]), new)
    page = torch.as_tensor(table[owner, place // PAGE], device=DEVICE).long()
    slot = torch.as_tensor(place % PAGE, device=DEVICE)
    kp.transpose(1, 2)[page, slot] = k
    vp.transpose(1, 2)[page, slot] = s["v"].double()
    return {"q": q, "k_pages": kp, "v_pages": vp, "new_prefix_len": _i32(before + new)}


def _sample_exact(s):
    x = s["logits"][:, :s["case"]["vocab"]].double().cpu().numpy()
    par = [s[name].cpu().numpy() for name in ("temperature", "top_k", "top_p", "min_p", "u")]
    return torch.as_tensor(np.array([_token_exact(*row) for row in zip(x, *par)], np.int32))


def _token_exact(row, t, k, p, least, u):
    if t == 0:
        return row.argmax()
    mass = np.rint(np.exp((row - row.max()) / np.float64(t)) * UNIT).astype(np.int64)
    order = np.lexsort((np.arange(row.size), -row))
    if k > 0:
        order = order[:k]
    if p < 1:
        upto = np.cumsum(mass[order])
        order = order[:max(1, int(np.searchsorted(upto - mass[order], np.float64(p) * np.float64(upto[-1]), "left")))]
    order = np.sort(order[mass[order] >= np.float64(least) * UNIT])
    upto = np.cumsum(mass[order])
    return order[np.searchsorted(upto, np.float64(u) * np.float64(upto[-1]), "right")]
