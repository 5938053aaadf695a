"""The serving operators at ends of what they take that serve no model today:
pages of any size, very many requests, rows and heads, scales of any sign."""
import numpy as np
import pytest

from oracle import serving
from paged_calls import check, run_decode, run_prompt
from serving_inputs import Cache, back, to_dev, typed
from test_gpu_append import close, inv_freq
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)
from test_gpu_sample import draw, parameters

pytestmark = pytest.mark.gpu


def append(ada, new, prefix, ps, hq, hkv, d, dtype, columns, holes=()):  # noqa: F811
    import torch
    rng = np.random.default_rng(ps + len(new))
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T, B = int(indptr[-1]), len(new)
    table = np.full((B, columns), -1, np.int32)
    order = rng.permutation(B * columns + 2)
    table[:] = order[:B * columns].reshape(B, columns)
    for r, e in holes:
        table[r, e] = -1
    pages = B * columns + 2
    rows = typed(rng.standard_normal((T, hq + 2 * hkv, d)), dtype)
    x = to_dev(rows)
    pool = typed(np.full((pages, hkv, ps, d), 77.0), dtype)
    kp, vp = to_dev(pool), to_dev(pool)
    q = torch.zeros((T, hq, d), dtype=x.dtype, device="cuda")
    grown = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    print("append tokens", T, "requests", B, "page size", ps, flush=True)
    ada.adaserve_rope_append_kv(token_indptr=to_dev(indptr), prefix_len=to_dev(np.asarray(prefix, np.int32)), q=x[:, :hq],
                                k=x[:, hq:hq + hkv], v=x[:, hq + hkv:], inv_freq=to_dev(inv_freq(d)), q_out=q, k_pages=kp,
                                v_pages=vp, block_table=to_dev(table), new_prefix_len=grown)
    torch.cuda.synchronize()
    req, place, page, new_len = serving.append_places(indptr, prefix, table, pages, ps, T)
    assert (req >= 0).all() and back(grown).tolist() == new_len.tolist()
    close(back(q), serving.rope(rows[:, :hq], place, inv_freq(d)), rows, dtype)
    gk, gv = back(kp), back(vp)
    at = np.flatnonzero(page >= 0)
    close(gk[page[at], :, place[at] % ps], serving.rope(rows[:, hq:hq + hkv], place, inv_freq(d))[at], rows, dtype)
    ek, ev = pool.copy(), pool.copy()
    ek[page[at], :, place[at] % ps] = gk[page[at], :, place[at] % ps]
    ev[page[at], :, place[at] % ps] = rows[at, hq + hkv:]
    assert gk.tobytes() == ek.tobytes() and gv.tobytes() == ev.tobytes()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps", [1, 5, 16, 64])
def test_append_page_sizes(ada, dtype, ps):  # noqa: F811
    new, prefix = [40, 0, 1, 77], [3, 9, 4, 0]
    append(ada, new, prefix, ps, 4, 2, 64, dtype, -(-80 // ps) + 1, holes=[(3, 50 // ps)])


def test_append_many_requests(ada):  # noqa: F811
    """More requests than 64^2 search steps, some without a token."""
    rng = np.random.default_rng(2)
    new = rng.integers(0, 3, 9000)
    append(ada, new, rng.integers(0, 9, 9000), 4, 2, 1, 64, "bf16", 3)


@pytest.mark.parametrize("scale", [-0.1, 0.0, 2.0])
def test_f32_scales(ada, scale):  # noqa: F811
    rng = np.random.default_rng(3)
    for new, ctx in (([70, 3, 33], [70, 1500, 40]), ([1, 1, 1, 1], [3000, 1, 0, 17])):
        c = Cache(rng, ctx, 2, 128, "f32")
        q = typed(rng.standard_normal((sum(new), 8, 128)), "f32")
        check("prompt", run_prompt(ada, q, new, ctx, c, "f32", scale), q, new, ctx, c, "f32", scale)
        if max(new) == 1:
            check("decode", run_decode(ada, q, ctx, c, "f32", scale), q, new, ctx, c, "f32", scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(4096, 4096), (4096, 256), (45, 3)])
def test_attention_many_heads(ada, dtype, hq, hkv):  # noqa: F811
    rng = np.random.default_rng(hkv)
    for new, ctx in (([5, 2], [5, 70]), ([1, 1], [300, 33])):
        c = Cache(rng, ctx, hkv, 64, dtype)
        q = typed(rng.standard_normal((sum(new), hq, 64)), dtype)
        check("prompt", run_prompt(ada, q, new, ctx, c, dtype, 0.125), q, new, ctx, c, dtype, 0.125)
        if max(new) == 1:
            check("decode", run_decode(ada, q, ctx, c, dtype, 0.125), q, new, ctx, c, dtype, 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_many_rows(ada, dtype):  # noqa: F811
    rng = np.random.default_rng(4)
    rows = 3000
    x = typed(rng.standard_normal((rows, 300)) * 2, dtype)
    draw(ada, x, 297, rng.random(rows), **parameters(rng, rows))
