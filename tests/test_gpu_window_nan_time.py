"""A key that is not a number costs a prompt over a window no more than its tiles done once again."""
import numpy as np
import pytest

import window_calls as calls
from paged_calls import starts
from serving_inputs import PS
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at", [2, 5000])
def test_rows_behind_it_are_not_taken_one_by_one(ada, dtype, at):  # noqa: F811
    """A sink, which all rows see, and a key that those of a window see: one by one they took hundreds of times a clean call."""
    import torch
    n, window, sinks, hq, hkv, d = 8192, 4096, 4, 8, 2, 128
    torch.manual_seed(at)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, v = (torch.randn(n // PS, hkv, PS, d, device="cuda").to(t) for _ in range(2))
    q = torch.randn(n, hq, d, device="cuda").to(t)
    out = torch.empty_like(q)
    indptr, ctx = starts([n]), np.array([n], np.int32)
    need = ada.adaserve_window_prompt_attn_workspace_bytes(indptr, ctx, hq, hkv, d, PS, window, sinks, calls.code(ada, dtype))
    args = dict(token_indptr=torch.from_numpy(indptr).cuda(), token_indptr_host=indptr, q=q, k_pages=k, v_pages=v, window=window,
                sinks=sinks, block_table=torch.arange(n // PS, dtype=torch.int32, device="cuda")[None], context_len_host=ctx,
                context_len=torch.from_numpy(ctx).cuda(), sm_scale=0.09, out=out, workspace=calls.workspace(need))

    def took():
        us = []
        for _ in range(4):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            ada.adaserve_window_prompt_attn(**args)
            b.record()
            torch.cuda.synchronize()
            us.append(a.elapsed_time(b))
        return min(us)

    clean = took()
    k[at // PS, :, at % PS] = float("nan")
    with_nan = took()
    print("clean", clean, "with a NaN", with_nan, "ms", flush=True)
    rows = out.isnan().all(2).all(1).cpu().numpy()
    pos = np.arange(n)
    sees = (pos >= at) & ((at < sinks) | (at > pos - window))
    assert np.array_equal(rows, sees) and not out[~torch.from_numpy(sees).cuda()].isnan().any()
    assert with_nan < 10 * clean
