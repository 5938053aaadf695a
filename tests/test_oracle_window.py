"""The fp64 oracle of the attention over a window and of the cache's pages,
pinned by dense masks, by hand and by what has to hold of any tables (CPU)."""
import numpy as np
import pytest

from oracle import serving, window as oracle
from window_calls import Cache, Trees, starts


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (5, 3), (16, 16), (1000, 0), (7, 1000)])
def test_paged_attention_is_a_masked_softmax(window, sinks):
    import torch
    rng = np.random.default_rng(1)
    new, ctx = [3, 0, 9], [30, 4, 9]
    cache = Cache(rng, ctx, 2, 64, "f32")
    q = rng.standard_normal((12, 4, 64)).astype(np.float32)
    out, _, _ = oracle.paged_attention(q, starts(new), cache.k, cache.v, cache.table, ctx, 0.125, window, sinks)
    row = 0
    for r, (n, c) in enumerate(zip(new, ctx)):
        place = np.arange(c)
        k, v = (x[cache.table[r][place // 16], :, place % 16].astype(np.float64) for x in (cache.k, cache.v))
        i, j = np.arange(c - n, c)[:, None], place[None, :]
        hidden = (j > i) | ((i - j >= window) & (j >= sinks))
        for h in range(4):
            z = torch.tensor(q[row:row + n, h].astype(np.float64) @ k[:, h // 2].T * 0.125)
            p = torch.softmax(z.masked_fill(torch.tensor(hidden), -np.inf), 1).numpy()
            assert np.allclose(out[row:row + n, h], p @ v[:, h // 2], atol=1e-12)
        row += n


def test_without_a_window_it_is_the_causal_oracle():
    rng = np.random.default_rng(2)
    new, ctx = [5, 8], [40, 8]
    cache = Cache(rng, ctx, 2, 64, "bf16")
    q = rng.standard_normal((13, 4, 64)).astype(np.float32)
    full = serving.paged_attention(q, starts(new), cache.k, cache.v, cache.table, ctx, 0.125)[0]
    for window, sinks in ((40, 0), (10 ** 6, 3), (1, 40)):
        assert np.allclose(oracle.paged_attention(q, starts(new), cache.k, cache.v, cache.table, ctx, 0.125, window, sinks)[0], full)


def test_a_chain_of_nodes_is_a_chunk_of_a_prompt():
    rng = np.random.default_rng(3)
    n, L = 20, 33
    cache = Cache(rng, [L + n], 2, 64, "f32")
    place = L + np.arange(n)
    trees = Trees(rng, [n], 2, 64, "f32", chain=True)
    trees.k, trees.v = (x[cache.table[0][place // 16], :, place % 16] for x in (cache.k, cache.v))
    q = rng.standard_normal((n, 4, 64)).astype(np.float32)
    for window, sinks in ((1, 0), (10, 2), (25, 40), (99, 0)):
        a = oracle.paged_attention(q, [0, n], cache.k, cache.v, cache.table, [L + n], 0.125, window, sinks)[0]
        b = oracle.tree_attention(q, trees.indptr, trees.parent, trees.k, trees.v, cache.k, cache.v, cache.table, [L], 0.125,
                                  window, sinks)[0]
        assert np.allclose(a, b, atol=1e-13)


def test_a_branch_sees_its_own_path():
    """Root and two children that differ in nothing but their own value."""
    q = np.zeros((3, 1, 64))
    v = np.zeros((3, 1, 64), np.float32)
    v[:, 0, 0] = [1, 10, 100]
    none = np.zeros((1, 1, 16, 64), np.float32)
    out = oracle.tree_attention(q, [0, 3], [-1, 0, 0], np.zeros_like(v), v, none, none, np.zeros((1, 1), np.int32), [0], 1.0, 2, 0)[0]
    assert out[:, 0, 0].tolist() == [1.0, 5.5, 50.5]
    out = oracle.tree_attention(q, [0, 3], [-1, 0, 0], np.zeros_like(v), v, none, none, np.zeros((1, 1), np.int32), [0], 1.0, 1, 0)[0]
    assert out[:, 0, 0].tolist() == [1.0, 10.0, 100.0]


def test_update_by_hand():
    table = np.array([[3, 1, 0, -1], [5, -1, -1, -1]], np.int32)
    refs = np.array([1, 1, 0, 1, 0, 2], np.int32)
    # row 0: 40 tokens, a window of 9 and 2 sinks: positions 32 .. 40 and 0, 1 are seen, so page 1 goes
    t, f, c = oracle.update_pages([40, 16], [50, 33], 9, 2, 16, table, refs)
    assert t.tolist() == [[3, -1, 0, 1], [5, 2, 4, -1]] and f.tolist() == [1, 1, 1, 1, 1, 2] and c.tolist() == [50, 33]
    t, f, c = oracle.update_pages([-1, 16], None, 9, 2, 16, table, refs)
    assert t.tolist() == [[-1] * 4, [5, -1, -1, -1]] and f.tolist() == [0, 0, 0, 0, 0, 2] and c is None


def test_fork_by_hand():
    table = np.array([[3, 1, 0], [5, 2, -1]], np.int32)
    refs = np.array([1, 1, 1, 1, 0, 1, 0], np.int32)
    t, n, f, a, b = oracle.fork_pages([1, 0, 1, 1], [20, 24], 16, table, refs)
    # row 0 goes to new row 1 with its spare page; row 1 to three rows, which share page 5
    assert t.tolist() == [[5, 2, -1], [3, 1, 0], [5, 4, -1], [5, 6, -1]] and n.tolist() == [24, 20, 24, 24]
    assert f.tolist() == [1, 1, 1, 1, 1, 3, 1] and a.tolist() == [-1, -1, 2, 2] and b.tolist() == [-1, -1, 4, 6]


def test_compact_by_hand():
    t, f, p, a, b, c = oracle.compact_pages(np.array([[4, 0, 9, 1]], np.int32), np.array([1, 0, 0, 2, 1], np.int32))
    assert t.tolist() == [[2, 0, 9, -1]] and f.tolist() == [1, 2, 1, 0, 0] and p.tolist() == [0, -1, -1, 1, 2]
    assert a.tolist() == [3, 4, -1, -1, -1] and b.tolist() == [1, 2, -1, -1, -1] and c.tolist() == [3, 2]


@pytest.mark.parametrize("seed", range(20))
def test_references_count_the_entries(seed):
    """Through updates, forks and compactions of caches whose pages nobody else keeps."""
    rng = np.random.default_rng(seed)
    B, stride, P, ps = int(rng.integers(1, 6)), int(rng.integers(1, 9)), int(rng.integers(1, 40)), int(rng.integers(1, 9))
    table, refs, lens = np.full((B, stride), -1, np.int32), np.zeros(P, np.int32), np.zeros(B, np.int64)
    for _ in range(12):
        need = np.minimum(lens + rng.integers(0, 3 * ps, B), stride * ps)
        gone = np.where(rng.random(B) < 0.1, -1, lens)
        table, refs, capacity = oracle.update_pages(gone, need, int(rng.integers(0, 20)), int(rng.integers(0, 4)), ps, table, refs)
        lens = np.where(gone < 0, 0, np.minimum(capacity, need))
        source = rng.integers(0, B, B)
        table, lens, refs, src, dst = oracle.fork_pages(source, lens, ps, table, refs)
        assert len(set(dst[dst >= 0].tolist())) == (dst >= 0).sum() and not set(dst[dst >= 0].tolist()) & set(src.tolist())
        table, refs, place, src, dst, counts = oracle.compact_pages(table, refs)
        assert (refs == np.bincount(table[table >= 0], minlength=P)).all()
        assert (refs[:counts[0]] > 0).all() and (refs[counts[0]:] == 0).all()
