"""GPU parity of adaserve_rope_append_kv with the fp64 oracle: rotated queries
and keys, the whole page pools and the new lengths."""
import numpy as np
import pytest

from oracle import serving
from serving_inputs import PS, Cache, back, to_dev, typed

pytestmark = pytest.mark.gpu

SENTINEL = 77.0


@pytest.fixture(scope="module")
def ada():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2501_12162_amd as ada
    ada.load_library()
    return ada


def inv_freq(rotary, theta=500000.0):
    return (theta ** (-np.arange(0, rotary, 2) / max(rotary, 1))).astype(np.float32)


def close(got, ref, x, dtype):
    """|error| <= half a step of the output plus what sine, cosine (2^-22.5 of
    angle reduction and evaluation) and the fp32 turn may add to each pair."""
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    bound = step * np.abs(ref) + 2.0 ** -21 * 2 * np.abs(serving.widen(x)).max(initial=0) + 1e-30
    bad = ~(np.abs(serving.widen(got) - ref) <= bound)
    assert not bad.any(), (np.abs(serving.widen(got) - ref)[bad].max(), bad.sum())


def run(ada, seed, new, prefix, hq=4, hkv=2, d=128, dtype="bf16", rotary=None, interleaved=False, fused=True, pad=0,
        reach=None, table=None, positions=None, in_place=False, append=True, want_k=False):
    import torch
    rng = np.random.default_rng(seed)
    new, prefix = np.asarray(new), np.asarray(prefix)
    rotary = d if rotary is None else rotary
    T = int(new.sum()) + pad
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    c = Cache(rng, np.maximum(prefix, 0), hkv, d, dtype, reach=np.maximum(prefix, 0) + new if reach is None else reach)
    table = c.table if table is None else table(c)
    rows = typed(rng.standard_normal((T, hq + 2 * hkv, d)), dtype)
    x = to_dev(rows)
    q, k, v = (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]) if fused else \
        tuple(t.contiguous() for t in (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]))
    inv = inv_freq(rotary)
    qo = q if in_place else torch.full((T, hq, d), SENTINEL, dtype=x.dtype, device="cuda")
    ko = (k if in_place else torch.full((T, hkv, d), SENTINEL, dtype=x.dtype, device="cuda")) if want_k else None
    kp, vp, plen = to_dev(c.k), to_dev(c.v), to_dev(prefix.astype(np.int32))
    new_len = plen if in_place else torch.full((len(new),), -9, dtype=torch.int32, device="cuda")
    print("append seed", seed, "tokens", T, "requests", len(new), flush=True)
    ada.adaserve_rope_append_kv(
        token_indptr=to_dev(indptr), prefix_len=plen, q=q, k=k, v=v if append else None,
        inv_freq=to_dev(inv) if rotary else None, interleaved=interleaved,
        positions=None if positions is None else to_dev(np.asarray(positions, np.int32)), q_out=qo, k_out=ko,
        k_pages=kp if append else None, v_pages=vp if append else None,
        block_table=to_dev(np.ascontiguousarray(table)) if append else None, new_prefix_len=new_len if append else None)
    torch.cuda.synchronize()
    req, place, page, grown = serving.append_places(indptr, prefix, table, c.pages, PS, T)
    own = req >= 0
    pos = place if positions is None else np.asarray(positions)
    rq, rk = (serving.rope(rows[:, a:b], pos, inv, interleaved) for a, b in ((0, hq), (hq, hq + hkv)))
    gq = back(qo)
    close(gq[own], rq[own], rows, dtype)
    old = rows[:, :hq] if in_place else typed(np.full((T, hq, d), SENTINEL), dtype)
    assert np.array_equal(gq[~own], old[~own])
    if want_k:
        close(back(ko)[own], rk[own], rows, dtype)
    gk, gv = back(kp), back(vp)
    if not append:
        assert gk.tobytes() == c.k.tobytes() and gv.tobytes() == c.v.tobytes()
        return
    assert back(new_len).tolist() == grown.tolist()
    stored = np.flatnonzero(page >= 0)
    ek, ev = c.k.copy(), c.v.copy()
    close(gk[page[stored], :, place[stored] % PS], rk[stored], rows, dtype)
    ek[page[stored], :, place[stored] % PS] = gk[page[stored], :, place[stored] % PS]
    ev[page[stored], :, place[stored] % PS] = rows[stored, hq + hkv:]
    assert gk.tobytes() == ek.tobytes() and gv.tobytes() == ev.tobytes()   # values bit for bit, nothing else touched
    return grown


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,prefix", [([1], [0]), ([1], [1500]), ([17, 1, 0, 40], [0, 15, 3, 16]), ([1] * 70, list(range(70))),
                                        ([700, 3, 600], [1, 100000, 31])])
def test_append(ada, dtype, new, prefix):
    # a far position needs no far pages: its prefix lies on pages that its table does not list
    far = np.minimum(prefix, 200)
    run(ada, len(new), new, far, dtype=dtype)
    t = np.concatenate([np.arange(p, p + n) for p, n in zip(prefix, new)])
    run(ada, len(new), new, far, dtype=dtype, positions=t)


@pytest.mark.parametrize("kw", [
    dict(rotary=0), dict(rotary=64), dict(rotary=16, interleaved=True), dict(interleaved=True), dict(d=64, hq=8, hkv=8),
    dict(d=256, hq=3, hkv=1), dict(d=512, dtype="f32", interleaved=True), dict(d=8, rotary=0), dict(d=80, rotary=48, hq=5, hkv=5),
    dict(fused=False), dict(fused=False, in_place=True, want_k=True), dict(pad=9), dict(want_k=True),
    dict(append=False, want_k=True), dict(append=False, want_k=True, pad=3, dtype="f32", rotary=64, interleaved=True),
])
def test_append_layouts(ada, kw):
    run(ada, 11, [5, 0, 33, 1], [0, 9, 14, 31], **kw)
    run(ada, 12, [400, 700, 1], [7, 16, 250], **kw)     # several tokens to a workgroup


def test_append_positions_beyond_fp32(ada):
    """Angles of far positions: fp32 would be off by 0.5 rad at 2^23."""
    pos = [0, 1, 65535, 100003, 2 ** 22 + 1, 2 ** 23 - 1, 2 ** 31 - 1, -5]
    for dtype in ("bf16", "f32"):
        run(ada, 3, [8], [0], dtype=dtype, positions=pos, append=False, want_k=True)


def test_append_missing_room(ada):
    """A table that ends, a hole, a page id outside the pool, a negative length:
    rows without a page are dropped, lengths count the leading rows."""
    def holes(c):
        t = c.table.copy()
        t[0, 1] = -1
        t[1, 0] = c.pages
        t[2, 2] = -7
        return t[:, :3]
    grown = run(ada, 5, [40, 4, 20, 3, 60], [0, 0, 16, -3, 16], reach=[40, 16, 48, 16, 48], table=holes)
    assert grown.tolist() == [16, 0, 32, -3, 48]


def test_append_replayed_from_a_graph(ada):
    """One captured decode step whose lengths grow in place: replays with the
    program's own work between them equal eager calls."""
    import torch
    rng = np.random.default_rng(9)
    B, hq, hkv, d = 5, 8, 2, 128
    start = np.array([0, 15, 16, 40, 3], np.int32)
    c = Cache(rng, start, hkv, d, "bf16", reach=start + 8)
    q, k, v = (to_dev(typed(rng.standard_normal((B, h, d)), "bf16")) for h in (hq, hkv, hkv))
    indptr, table, inv = to_dev(np.arange(B + 1, dtype=np.int32)), to_dev(c.table), to_dev(inv_freq(d))

    def state():
        return [to_dev(c.k), to_dev(c.v), to_dev(start), torch.zeros_like(q)]

    def step(s):
        ada.adaserve_rope_append_kv(token_indptr=indptr, prefix_len=s[2], q=q, k=k, v=v, inv_freq=inv, q_out=s[3],
                                    k_pages=s[0], v_pages=s[1], block_table=table, new_prefix_len=s[2])
    eager, graphed = state(), state()
    warm = state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(graphed)
    for rep in range(4):
        q.copy_(torch.randn_like(q))
        k.copy_(torch.randn_like(k))
        step(eager)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, graphed):
            assert back(a).tobytes() == back(b).tobytes(), rep
        assert eager[2].tolist() == (start + rep + 1).tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", ["q", "k"])
def test_queries_or_keys_alone(ada, dtype, which):
    """Rows of one kind only: no pages, no other output."""
    import torch
    rng = np.random.default_rng(17)
    new, prefix, h, d = [3, 0, 1200], [5, 2, 31], 6, 128
    indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    x = typed(rng.standard_normal((int(indptr[-1]) + 2, h, d)), dtype)
    inv = inv_freq(d)
    out = torch.full(x.shape, SENTINEL, dtype=to_dev(x[:1]).dtype, device="cuda")
    print("alone", which, dtype, flush=True)
    ada.adaserve_rope_append_kv(token_indptr=to_dev(indptr), prefix_len=to_dev(np.asarray(prefix, np.int32)),
                                inv_freq=to_dev(inv), **{which: to_dev(x), which + "_out": out})
    torch.cuda.synchronize()
    req, place, _, _ = serving.append_places(indptr, prefix, np.zeros((3, 0), np.int32), 0, PS, len(x))
    own = req >= 0
    close(back(out)[own], serving.rope(x, place, inv)[own], x, dtype)
    assert (serving.widen(back(out)[~own]) == SENTINEL).all()
