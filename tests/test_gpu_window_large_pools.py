"""Pools whose far pages lie past 2^32 bytes: pages copied there, and the attentions over a window
reading them, give what the same pages give at the front."""
import numpy as np
import pytest

import window_calls as calls
from paged_calls import starts
from serving_inputs import PS, to_dev
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
D, HQ, HKV, WINDOW, SINKS, SCALE = 128, 8, 8, 1500, 20, 0.09
NEW, CTX = {"prompt": [40, 70], "decode": [1, 1], "tree": [9, 20]}, [900, 2100]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["prompt", "decode", "tree"])
def test_far_pages(ada, kind, dtype):  # noqa: F811
    import torch
    rng = np.random.default_rng(40)
    new, ctx = NEW[kind], np.asarray(CTX, np.int32)
    cache, trees, q = calls.case(rng, kind, dtype, D, HQ, HKV, new, CTX, WINDOW, SINKS)
    near = cache.pages
    page_bytes = HKV * PS * D * (2 if dtype == "bf16" else 4)
    far = 2 ** 32 // page_bytes + 5
    k, v = (torch.zeros(far + near, HKV, PS, D, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
            for _ in range(2))
    k[:near], v[:near] = to_dev(cache.k), to_dev(cache.v)
    order = torch.arange(near, dtype=torch.int32, device="cuda")
    print("far pages", kind, dtype, "from", far, "of", page_bytes, "bytes", flush=True)
    ada.adaserve_copy_pages(src=order, dst=order + far, k_pages=k, v_pages=v)
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    for pool in (k, v):
        assert torch.equal(pool[far:].view(bits), pool[:near].view(bits)) and not pool[near:far:997].any()
    indptr, code = starts(new), calls.code(ada, dtype)
    args = dict(q=to_dev(q), k_pages=k, v_pages=v, window=WINDOW, sinks=SINKS, sm_scale=SCALE)
    shape = (HQ, HKV, D, PS, WINDOW, SINKS, code)
    query = getattr(ada, "adaserve_window_%s_attn_workspace_bytes" % kind)
    if kind == "decode":
        args.update(context_len=to_dev(ctx), max_context=max(CTX), workspace=calls.workspace(query(len(CTX), max(CTX), *shape)))
    elif kind == "prompt":
        args.update(token_indptr=to_dev(indptr), token_indptr_host=indptr, context_len=to_dev(ctx), context_len_host=ctx,
                    workspace=calls.workspace(query(indptr, ctx, *shape)))
    else:
        args.update(node_indptr=to_dev(indptr), node_indptr_host=indptr, parent=to_dev(trees.parent), prefix_len=to_dev(ctx),
                    prefix_len_host=ctx, k_tree=to_dev(trees.k), v_tree=to_dev(trees.v),
                    workspace=calls.workspace(query(indptr, ctx, *shape)))
    outs = []
    for shift in (0, far):
        table = np.where((cache.table >= 0) & (cache.table < near), cache.table + shift, -1).astype(np.int32)
        out = torch.full(q.shape, 7, dtype=k.dtype, device="cuda")
        getattr(ada, "adaserve_window_%s_attn" % kind)(block_table=to_dev(table), out=out, **args)
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.equal(outs[0].view(bits), outs[1].view(bits))
    got = calls.widen(outs[0].cpu().view(bits).numpy().view(np.uint16) if dtype == "bf16" else outs[0].cpu().numpy())
    calls.check(kind, dtype, got, calls.expected(kind, cache, trees, q, new, CTX, SCALE, WINDOW, SINKS), max(CTX) + 40)
