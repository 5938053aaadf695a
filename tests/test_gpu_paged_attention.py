"""GPU parity of adaserve_prompt_attn and adaserve_decode_attn with the fp64
oracle, at the lengths, heads and masks where they can go wrong."""
import numpy as np
import pytest

from oracle import serving
from serving_inputs import PS, Cache, attention_bound, back, to_dev, typed

pytestmark = pytest.mark.gpu

SENTINEL = 77.0


@pytest.fixture(scope="module")
def ada():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2501_12162_amd as ada
    ada.load_library()
    return ada


def code(ada, dtype):
    return ada.ADASERVE_BF16 if dtype == "bf16" else ada.ADASERVE_F32


def check(got, ref, dtype, keys, d):
    out, size, reach = ref
    got = serving.widen(got)
    assert np.isfinite(got).all()
    bound = attention_bound(dtype, out, size, reach, keys, d)
    err = np.abs(got - out)
    assert (err <= bound).all(), (float((err / bound).max()), float(err.max()))


def rows_of(rng, T, hq, d, dtype, strided):
    """Query rows, dense or as the first part of wider rows."""
    x = typed(rng.standard_normal((T, hq + (2 if strided else 0), d)), dtype)
    return x[:, :hq], to_dev(x)[:, :hq]


def prompt(ada, seed, new, ctx, hq=8, hkv=2, d=128, dtype="bf16", pad=0, strided=False, scale=None, table=None, edit=None):
    import torch
    rng = np.random.default_rng(seed)
    new, ctx = np.asarray(new), np.asarray(ctx)
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(indptr[-1])
    c = Cache(rng, ctx, hkv, d, dtype)
    if table is not None:
        c.table = table(c)
    if edit is not None:
        edit(c)
    qh, q = rows_of(rng, T + pad, hq, d, dtype, strided)
    scale = d ** -0.5 if scale is None else scale
    ctx32 = ctx.astype(np.int32)
    need = ada.adaserve_prompt_attn_workspace_bytes(indptr, ctx32, hq, hkv, d, PS, code(ada, dtype))
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    out = torch.full((T + pad, hq, d), SENTINEL, dtype=q.dtype, device="cuda")
    print("prompt seed", seed, "rows", T, "longest", int(ctx.max(initial=0)), "workspace", need, flush=True)
    ada.adaserve_prompt_attn(token_indptr=to_dev(indptr), token_indptr_host=indptr, q=q, k_pages=to_dev(c.k),
                             v_pages=to_dev(c.v), block_table=to_dev(c.table), context_len=to_dev(ctx32),
                             context_len_host=ctx32, sm_scale=scale, out=out, workspace=ws)
    torch.cuda.synchronize()
    got = back(out)
    assert (serving.widen(got[T:]) == SENTINEL).all()   # padding rows are left as they were
    ref = serving.paged_attention(qh[:T], indptr, c.k, c.v, c.table, ctx, scale)
    check(got[:T], ref, dtype, int(ctx.max(initial=0)), d)
    return got


HEADS = [(8, 2), (4, 4), (16, 1), (6, 2), (7, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,ctx", [
    ([1], [1]), ([1], [17]), ([2, 0, 3], [2, 5, 3]), ([15, 16, 17], [15, 16, 17]), ([31, 32, 33], [31, 32, 33]),
    ([63, 64, 65, 1], [63, 64, 65, 1]), ([127, 129], [127, 129]), ([300], [300]), ([5, 40], [100, 1000]),
    ([130, 1, 7], [131, 700, 2000]),
])
def test_prompt_lengths(ada, dtype, new, ctx):
    prompt(ada, sum(ctx), new, ctx, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", HEADS)
def test_prompt_heads(ada, dtype, d, hq, hkv):
    prompt(ada, hq * 10 + hkv, [37, 3, 90], [37, 50, 101], hq=hq, hkv=hkv, d=d, dtype=dtype, strided=True, pad=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_rows_that_see_nothing(ada, dtype):
    """Fewer cached keys than rows (an append that found no room): the rows
    before position 0 give zeros; no key at all gives zeros throughout."""
    got = prompt(ada, 3, [40, 5, 70, 3], [33, 0, 1, 3], dtype=dtype)
    assert not serving.widen(got[:7]).any() and not serving.widen(got[40:45]).any()
    assert not serving.widen(got[45:114]).any() and serving.widen(got[114]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_pages_outside_the_pool(ada, dtype):
    """Entries outside the pool are all-zero pages (score 0, value 0)."""
    def holes(c):
        t = c.table.copy()
        t[0, 1], t[0, 4], t[1, 0] = -1, c.pages, 2 ** 31 - 1
        return t
    prompt(ada, 4, [90, 20], [90, 45], dtype=dtype, table=holes)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan, 3.3e38, -3.3e38])
def test_prompt_keys_that_a_row_does_not_see(ada, dtype, bad):
    """What stands behind a row's position does not reach it: the last tokens'
    keys and values are infinite, NaN or the type's largest, and the rows before
    them come out as ever."""
    import torch
    n, hidden = 150, 20

    def run(poison):
        rng = np.random.default_rng(8)
        c = Cache(rng, [n], 2, 128, dtype)
        if poison:
            for t in range(n - hidden, n):
                c.k[c.table[0, t // PS], :, t % PS] = typed(np.full(128, bad), dtype)
                c.v[c.table[0, t // PS], :, t % PS] = typed(np.full(128, bad), dtype)
        q = to_dev(typed(np.random.default_rng(9).standard_normal((n, 8, 128)), dtype))
        out = torch.empty_like(q)
        indptr, ctx = np.array([0, n], np.int32), np.array([n], np.int32)
        ada.adaserve_prompt_attn(token_indptr=to_dev(indptr), token_indptr_host=indptr, q=q, k_pages=to_dev(c.k),
                                 v_pages=to_dev(c.v), block_table=to_dev(c.table), context_len=to_dev(ctx),
                                 context_len_host=ctx, sm_scale=128 ** -0.5, out=out)
        torch.cuda.synchronize()
        return back(out), c, back(q)
    got, c, q = run(True)
    ref = serving.paged_attention(q[:n - hidden], [0, n - hidden], c.k, c.v, c.table, [n - hidden], 128 ** -0.5)
    check(got[:n - hidden], ref, dtype, n, 128)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,ctx", [([200], [260]), ([70], [1500]), ([600, 33], [601, 1200])])
def test_prompt_large_scores(ada, dtype, new, ctx):
    """Scores to the hundreds, rising and falling along the keys."""
    def steep(c):
        k = serving.widen(c.k)
        for row in c.table:
            for e, p in enumerate(row):
                if p >= 0:
                    k[p] *= (1 + e % 7 + (e > 60) * 9) * (-1) ** e
        c.k = typed(k, dtype)
    prompt(ada, 6, new, ctx, dtype=dtype, scale=1.0, edit=steep)


@pytest.mark.parametrize("seed", range(10))
def test_prompt_drawn(ada, seed):
    rng = np.random.default_rng(100 + seed)
    B = int(rng.integers(1, 7))
    new = rng.integers(0, int(rng.choice([3, 40, 300])), B)
    ctx = np.maximum(new + rng.integers(0, int(rng.choice([1, 20, 800])), B) - (rng.random(B) < 0.1) * 5, 0)
    hq, hkv = HEADS[int(rng.integers(len(HEADS)))]
    prompt(ada, seed, new, ctx, hq=hq, hkv=hkv, d=int(rng.choice([64, 128])), dtype=str(rng.choice(["bf16", "f32"])),
           strided=bool(rng.integers(2)), pad=int(rng.integers(0, 3)))


def test_prompt_chunks_equal_the_whole(ada):
    """A prompt in chunks over what is cached of it equals the prompt at once,
    within the roundings of both."""
    rng = np.random.default_rng(21)
    n, hq, hkv, d = 500, 8, 2, 128
    c = Cache(rng, [n], hkv, d, "bf16")
    q = to_dev(typed(rng.standard_normal((n, hq, d)), "bf16"))
    kp, vp, table = to_dev(c.k), to_dev(c.v), to_dev(c.table)
    import torch

    def part(a, b):
        indptr, ctx = np.array([0, b - a], np.int32), np.array([b], np.int32)
        out = torch.empty(b - a, hq, d, dtype=q.dtype, device="cuda")
        need = ada.adaserve_prompt_attn_workspace_bytes(indptr, ctx, hq, hkv, d, PS, ada.ADASERVE_BF16)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        ada.adaserve_prompt_attn(token_indptr=to_dev(indptr), token_indptr_host=indptr, q=q[a:b], k_pages=kp, v_pages=vp,
                                 block_table=table, context_len=to_dev(ctx), context_len_host=ctx, sm_scale=d ** -0.5,
                                 out=out, workspace=ws)
        torch.cuda.synchronize()
        return serving.widen(back(out))
    whole = part(0, n)
    pieces = np.concatenate([part(a, b) for a, b in ((0, 1), (1, 130), (130, 499), (499, 500))])
    ref, size, reach = serving.paged_attention(back(q), [0, n], c.k, c.v, c.table, [n], d ** -0.5)
    bound = attention_bound("bf16", ref, size, reach, n, d)
    assert (np.abs(whole - ref) <= bound).all() and (np.abs(pieces - ref) <= bound).all()


# ---- single tokens ----

def decode(ada, seed, ctx, hq=8, hkv=2, d=128, dtype="bf16", strided=False, most=None, table=None, scale=None):
    import torch
    rng = np.random.default_rng(seed)
    ctx = np.asarray(ctx)
    B = len(ctx)
    c = Cache(rng, np.maximum(ctx, 0), hkv, d, dtype)
    if table is not None:
        c.table = table(c)
    most = int(ctx.max()) if most is None else most
    if c.table.shape[1] * PS < most:
        c.table = np.concatenate([c.table, np.full((B, -(-most // PS) - c.table.shape[1]), -1, np.int32)], 1)
    qh, q = rows_of(rng, B, hq, d, dtype, strided)
    scale = d ** -0.5 if scale is None else scale
    need = ada.adaserve_decode_attn_workspace_bytes(B, most, hq, hkv, d, PS, code(ada, dtype))
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    out = torch.full((B, hq, d), SENTINEL, dtype=q.dtype, device="cuda")
    print("decode seed", seed, "requests", B, "longest", int(ctx.max()), "workspace", need, flush=True)
    ada.adaserve_decode_attn(q=q, k_pages=to_dev(c.k), v_pages=to_dev(c.v), block_table=to_dev(c.table),
                             context_len=to_dev(ctx.astype(np.int32)), max_context=most, sm_scale=scale, out=out,
                             workspace=ws)
    torch.cuda.synchronize()
    got = back(out)
    ok = (ctx >= 0) & (ctx <= most)
    assert np.isnan(serving.widen(got[~ok])).all()
    lens = np.where(ok, ctx, 0)
    o, s, reach = serving.paged_attention(qh, np.arange(B + 1), c.k, c.v, c.table, lens, scale)
    check(got[ok], (o[ok], s[ok], reach), dtype, int(lens.max()), d)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx", [[1], [2], [16, 17, 0, 31], [32, 33, 63, 64, 65], [1500], [4097, 1, 300], [0], [0, 0, 5],
                                 [128, 129, 255, 256, 257, 511, 512, 513], [9000]])
def test_decode_lengths(ada, dtype, ctx):
    decode(ada, sum(ctx), ctx, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", HEADS + [(32, 8)])
def test_decode_heads(ada, dtype, d, hq, hkv):
    decode(ada, hq * 10 + hkv, [700, 3, 0, 90, 1200], hq=hq, hkv=hkv, d=d, dtype=dtype, strided=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_many_requests(ada, dtype):
    rng = np.random.default_rng(5)
    decode(ada, 5, rng.integers(0, 90, 300), hq=4, hkv=2, d=64, dtype=dtype)
    decode(ada, 6, np.concatenate([rng.integers(0, 60, 90), [3000]]), hq=4, hkv=1, d=128, dtype=dtype)


@pytest.mark.parametrize("most", [100, 5000, 131072])
def test_decode_bounds_above_the_lengths(ada, most):
    decode(ada, 7, [100, 3, 0, 64], most=most)


def test_decode_lengths_outside_the_bound(ada):
    decode(ada, 8, [100, 41, -1, 40, 0], most=40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_pages_outside_the_pool(ada, dtype):
    def holes(c):
        t = c.table.copy()
        t[0, 1], t[0, 4], t[1, 0] = -1, c.pages, -2 ** 31
        return t
    decode(ada, 9, [90, 20, 700], dtype=dtype, table=holes)


@pytest.mark.parametrize("seed", range(8))
def test_decode_drawn(ada, seed):
    rng = np.random.default_rng(300 + seed)
    B = int(rng.integers(1, 20))
    ctx = rng.integers(0, int(rng.choice([20, 300, 6000])), B)
    hq, hkv = HEADS[int(rng.integers(len(HEADS)))]
    decode(ada, seed, ctx, hq=hq, hkv=hkv, d=int(rng.choice([64, 128])), dtype=str(rng.choice(["bf16", "f32"])),
           strided=bool(rng.integers(2)), most=int(ctx.max()) + int(rng.choice([0, 1, 1000])))


def test_decode_replayed_from_a_graph_with_growing_lengths(ada):
    """A captured call replayed while the lengths on the device grow, with
    eager work of another batch in another workspace between the replays."""
    import torch
    rng = np.random.default_rng(31)
    hq, hkv, d, most = 8, 2, 128, 2048
    c = Cache(rng, [most] * 4, hkv, d, "bf16")
    q = to_dev(typed(rng.standard_normal((4, hq, d)), "bf16"))
    kp, vp, table = to_dev(c.k), to_dev(c.v), to_dev(c.table)
    need = ada.adaserve_decode_attn_workspace_bytes(4, most, hq, hkv, d, PS, ada.ADASERVE_BF16)
    lens = to_dev(np.zeros(4, np.int32))

    def call(out, ws, lens):
        ada.adaserve_decode_attn(q=q, k_pages=kp, v_pages=vp, block_table=table, context_len=lens, max_context=most,
                                 sm_scale=d ** -0.5, out=out, workspace=ws)
    ws = [torch.empty(max(need, 1), dtype=torch.uint8, device="cuda") for _ in range(2)]
    out, eager = torch.empty_like(q), torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, ws[0], lens)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out, ws[0], lens)
    for now in ([1, 2, 3, 4], [100, 0, 2000, 31], [2048, 2048, 2048, 2048], [5, 1999, 700, 33]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        call(eager, ws[1], lens)
        torch.cuda.synchronize()
        assert back(out).tobytes() == back(eager).tobytes()
        o, s, reach = serving.paged_attention(back(q), np.arange(5), c.k, c.v, c.table, now, d ** -0.5)
        check(back(out), (o, s, reach), "bf16", most, d)
