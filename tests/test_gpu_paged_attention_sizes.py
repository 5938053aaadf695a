"""GPU parity of prompt and decode attention with the fp64 oracle at the sizes
that take other paths through the kernels: more tiles than workgroups, more
requests than a launch's table holds, contexts whose page ids are loaded in
several goes, split keys with hidden infinities, more requests than the decode
schedule deals out, and shares of it that hold many requests."""
import numpy as np
import pytest

from oracle import serving
from serving_inputs import PS, Cache, to_dev, typed
from test_gpu_paged_attention import ada, check, decode, prompt  # noqa: F401  (a fixture)

import test_gpu_paged_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("before", [0, 100])
def test_prompt_more_tiles_than_workgroups(ada, d, before):
    """576 tiles and more of 256 rows on 256 workgroups, with the same keys before every prompt."""
    new = np.array([1100, 1030, 1200, 1025, 1, 1100, 1290, 1111, 1040])
    prompt(ada, d + before, new, new + before, hq=16, hkv=4, d=d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_many_requests(ada, dtype):
    """More requests than the table of a launch takes, some of them empty."""
    rng = np.random.default_rng(11)
    new = rng.integers(0, 40, 200)
    new[rng.random(200) < 0.2] = 0
    prompt(ada, 11, new, new + rng.integers(0, 60, 200), hq=4, hkv=2, d=64, dtype=dtype)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("new,ctx", [([70], [2048]), ([33], [2049]), ([3, 65], [4096, 4161]), ([257], [6500])])
def test_prompt_long_contexts(ada, dtype, d, new, ctx):
    prompt(ada, sum(ctx), new, ctx, hq=4, hkv=2, d=d, dtype=dtype)


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_long_rows_and_contexts(ada, d):
    """Enough tiles that keys are not split, over more than one load of page ids."""
    need = ada.adaserve_prompt_attn_workspace_bytes(np.array([0, 2100], np.int32), np.array([4250], np.int32), 16, 4, d, PS,
                                                    ada.ADASERVE_BF16)
    assert need == 0
    prompt(ada, d, [2100], [4250], hq=16, hkv=4, d=d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,ctx,hq", [([40], [3300], 4), ([1300], [3300], 16)])
def test_prompt_pages_missing_in_long_contexts(ada, dtype, new, ctx, hq):
    """Pages outside the pool among the first page ids, the later ones, and the rows' own."""
    def holes(c):
        t = c.table.copy()
        for e in (0, 5, 63, 64, 126, 129, 130, 200):
            t[0, e] = -1 if e % 2 else c.pages
        t[0, -(-ctx[0] // PS) - 2] = -1
        return t
    prompt(ada, new[0], new, ctx, hq=hq, hkv=hq // 4, dtype=dtype, table=holes)


@pytest.mark.parametrize("bad", [np.inf, np.nan, 3.3e38])
def test_prompt_split_keys_that_a_row_does_not_see(ada, bad):
    """Keys split over workgroups, the last 20 keys and values infinite, NaN or the largest: the rows before them do not
    see them."""
    import torch
    n, ctx, hidden, hq, hkv, d = 120, 4000, 20, 8, 2, 128
    rng = np.random.default_rng(8)
    c = Cache(rng, [ctx], hkv, d, "bf16")
    for t in range(ctx - hidden, ctx):
        c.k[c.table[0, t // PS], :, t % PS] = typed(np.full(d, bad), "bf16")
        c.v[c.table[0, t // PS], :, t % PS] = typed(np.full(d, bad), "bf16")
    qh = typed(rng.standard_normal((n, hq, d)), "bf16")
    q = to_dev(qh)
    out = torch.empty_like(q)
    indptr, lens = np.array([0, n], np.int32), np.array([ctx], np.int32)
    need = ada.adaserve_prompt_attn_workspace_bytes(indptr, lens, hq, hkv, d, PS, ada.ADASERVE_BF16)
    assert need > 0
    ada.adaserve_prompt_attn(token_indptr=to_dev(indptr), token_indptr_host=indptr, q=q, k_pages=to_dev(c.k),
                             v_pages=to_dev(c.v), block_table=to_dev(c.table), context_len=to_dev(lens),
                             context_len_host=lens, sm_scale=d ** -0.5, out=out,
                             workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    m = n - hidden
    ref = serving.paged_attention(qh[:m], [0, m], c.k, c.v, c.table, [ctx - hidden], d ** -0.5)
    check(test_gpu_paged_attention.back(out)[:m], ref, "bf16", ctx, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_more_requests_than_are_dealt_out(ada, dtype, d):
    """1100 requests are a unit each; 1024 are dealt out."""
    rng = np.random.default_rng(12)
    for B in (1100, 1024):
        decode(ada, B, rng.integers(0, 200, B), hq=4, hkv=2, d=d, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_shares_of_many_requests(ada, dtype):
    """Mostly empty requests, also at both ends and between two shares; short ones beside one long one."""
    rng = np.random.default_rng(13)
    ctx = np.where(rng.random(700) < 0.8, 0, rng.integers(1, 300, 700))
    ctx[:5] = ctx[-7:] = 0
    decode(ada, 13, ctx, hq=4, hkv=4, dtype=dtype)
    ctx[350] = 20000
    decode(ada, 14, ctx, hq=8, hkv=1, dtype=dtype)
    decode(ada, 15, [128] * 64 + [0] * 3 + [256] * 64 + [0, 0], hq=8, hkv=8, d=64, dtype=dtype)


def test_decode_many_kv_heads(ada):
    """More kv-heads than workgroups on the device: one share holds the batch."""
    decode(ada, 16, [300, 0, 17, 150], hq=600, hkv=600, d=64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_pages_missing_in_long_contexts(ada, dtype):
    def holes(c):
        t = c.table.copy()
        for e in (0, 63, 64, 300, 511, 600):
            t[1, e] = -1 if e % 2 else c.pages
        return t
    decode(ada, 17, [20, 9700, 300], hq=4, hkv=1, dtype=dtype, table=holes)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pools_beyond_4_gib(ada, dtype):
    """Pages at the far end of pools of more than 2^32 bytes: what is appended there and read back by prompts and single
    tokens equals the same on the first pages, bit for bit."""
    import torch
    hq, hkv, d, new, ctx = 16, 8, 128, [40, 1], [70, 33]
    size = 2 if dtype == "bf16" else 4
    pages = 2 ** 32 // (hkv * PS * d * size) + 2000
    rng = np.random.default_rng(20)
    before = np.asarray(ctx) - new
    need = [-(-c // PS) for c in ctx]
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(indptr[-1])
    x = to_dev(typed(rng.standard_normal((T, hq + 2 * hkv, d)), dtype))
    old = [to_dev(typed(rng.standard_normal((sum(need), hkv, PS, d)), dtype)) for _ in range(2)]
    lens32, before32 = np.asarray(ctx, np.int32), before.astype(np.int32)
    pools = [torch.empty((pages, hkv, PS, d), dtype=x.dtype, device="cuda") for _ in range(2)]
    outs = []
    for first in (0, pages - sum(need)):
        table = np.full((2, max(need) + 1), -1, np.int32)
        at = first
        for r, n in enumerate(need):
            table[r, :n] = np.arange(at, at + n)
            at += n
        for pool, rows in zip(pools, old):
            pool[first:first + sum(need)] = rows
        table = to_dev(table)
        q = torch.empty((T, hq, d), dtype=x.dtype, device="cuda")
        grown = torch.empty(2, dtype=torch.int32, device="cuda")
        print("pools", dtype, "pages from", first, flush=True)
        ada.adaserve_rope_append_kv(token_indptr=to_dev(indptr), prefix_len=to_dev(before32), q=x[:, :hq], k=x[:, hq:hq + hkv],
                                    v=x[:, hq + hkv:], inv_freq=to_dev(np.ones(d // 2, np.float32)), q_out=q,
                                    k_pages=pools[0], v_pages=pools[1], block_table=table, new_prefix_len=grown)
        assert grown.tolist() == ctx
        kind = ada.ADASERVE_BF16 if dtype == "bf16" else ada.ADASERVE_F32
        prompts, singles = torch.empty_like(q), torch.empty_like(q[:2])
        for bytes_, call in (
                (ada.adaserve_prompt_attn_workspace_bytes(indptr, lens32, hq, hkv, d, PS, kind),
                 lambda ws: ada.adaserve_prompt_attn(
                     token_indptr=to_dev(indptr), token_indptr_host=indptr, q=q, k_pages=pools[0], v_pages=pools[1],
                     block_table=table, context_len=grown, context_len_host=lens32, sm_scale=d ** -0.5, out=prompts, workspace=ws)),
                (ada.adaserve_decode_attn_workspace_bytes(2, 96, hq, hkv, d, PS, kind),
                 lambda ws: ada.adaserve_decode_attn(
                     q=q[:2], k_pages=pools[0], v_pages=pools[1], block_table=torch.cat([table, table], 1), context_len=grown,
                     max_context=96, sm_scale=d ** -0.5, out=singles, workspace=ws))):
            call(torch.empty(max(bytes_, 1), dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        outs.append([test_gpu_paged_attention.back(t).tobytes() for t in
                     (prompts, singles, pools[0][first:first + sum(need)], pools[1][first:first + sum(need)])])
    assert outs[0] == outs[1]
