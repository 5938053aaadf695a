"""The pages of the cache: freed and taken, shared and copied, moved, against
plain loops over the same tables."""
import numpy as np
import pytest

from oracle import window as oracle
from serving_inputs import back, to_dev
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def i32(x):
    return np.asarray(x, np.int32)


def tables(rng, rows, stride, pages, lens, ps, extra=0.0, spare=0):
    """Rows with pages of their own for `lens` positions (and `spare` entries more), as far as there are pages, some of which
    other programs keep too; entries behind hold -1 or numbers outside the pool."""
    table = np.where(rng.random((rows, stride)) < 0.7, -1, pages + 3).astype(np.int32)
    perm = list(rng.permutation(pages))
    refs = np.zeros(pages, np.int32)
    for r in range(rows):
        for e in range(min(stride, -(-int(lens[r]) // ps) + spare)):
            if perm:
                table[r, e] = perm.pop()
                refs[table[r, e]] = 1
    refs[rng.random(pages) < extra] += 1
    return table, refs


def dev_workspace(ada, rows, pages):  # noqa: F811
    import torch
    return torch.full((ada.adaserve_pages_workspace_bytes(rows, pages),), 255, dtype=torch.uint8, device="cuda")


def empty(*shape):
    import torch
    return torch.full(shape, -99, dtype=torch.int32, device="cuda")


def update(ada, lens, need, window, sinks, ps, table, refs, in_place):  # noqa: F811
    import torch
    B, stride = table.shape
    bt, rf, cap = to_dev(table), to_dev(refs), empty(B) if need is not None else None
    nbt, nrf = (None, None) if in_place else (empty(B, stride), empty(len(refs)))
    print("update rows", B, stride, "pages", len(refs), "ps", ps, "window", window, sinks, in_place, flush=True)
    ada.adaserve_update_pages(context_len=to_dev(i32(lens)), need_len=None if need is None else to_dev(i32(need)), window=window,
                              sinks=sinks, page_size=ps, block_table=bt, page_refs=rf, new_block_table=nbt, new_page_refs=nrf,
                              capacity=cap, workspace=dev_workspace(ada, B, len(refs)))
    torch.cuda.synchronize()
    if not in_place:
        assert np.array_equal(back(bt), table) and np.array_equal(back(rf), refs)
        bt, rf = nbt, nrf
    return back(bt), back(rf), None if cap is None else back(cap)


def same(got, expected):
    for x, y in zip(got, expected):
        assert (x is None) == (y is None) and (x is None or np.array_equal(x, y)), (x, y)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows,stride,pages,ps,window,sinks,grow", [
    (1, 1, 1, 16, 1, 0, 1), (5, 20, 60, 16, 64, 4, 1), (7, 33, 400, 16, 100, 40, 200), (3, 600, 900, 16, 0, 0, 5000),
    (40, 50, 900, 16, 33, 1, 400), (4, 9, 30, 1, 3, 2, 4), (6, 300, 20000, 7, 50, 5, 2100), (2, 5000, 40000, 16, 4096, 4, 70000),
    (1500, 6, 3000, 16, 20, 4, 90), (20, 40, 300, 16, 2 ** 31 - 1, 0, 300), (20, 40, 300, 16, 5, 2 ** 31 - 1, 300),
    (64, 96, 8192, 16, 100, 4, 900), (64, 96, 8193, 16, 100, 4, 900), (65, 90, 4000, 16, 100, 4, 300), (64, 97, 4000, 16, 100, 4, 300),
])
def test_update(ada, rows, stride, pages, ps, window, sinks, grow, in_place):  # noqa: F811
    rng = np.random.default_rng([rows, stride, pages, window % 1000])
    lens = rng.integers(0, stride * ps + 1, rows) if rows > 1 else np.array([0])
    table, refs = tables(rng, rows, stride, pages, lens, ps, extra=0.05)
    need = np.minimum(lens + rng.integers(0, grow + 1, rows), stride * ps + 3)
    lens = np.where(rng.random(rows) < 0.2, -1, lens) if rows > 1 else lens
    got = update(ada, lens, need, window, sinks, ps, table, refs, in_place)
    same(got, oracle.update_pages(lens, need, window, sinks, ps, table, refs))


def test_update_frees_alone(ada):  # noqa: F811
    rng = np.random.default_rng(1)
    lens = rng.integers(0, 400, 9)
    table, refs = tables(rng, 9, 30, 200, lens, 16)
    lens[4] = -1
    for in_place in (False, True):
        same(update(ada, lens, None, 60, 4, 16, table, refs, in_place), oracle.update_pages(lens, None, 60, 4, 16, table, refs))


def test_update_of_shared_and_repeated_pages(ada):  # noqa: F811
    """Rows that share pages, a row that holds a page twice, a page that loses its last reference in this call and is taken in it,
    and pages that somebody else keeps."""
    table = i32([[0, 1, 2, -1], [0, 1, 3, -1], [5, 5, 4, -1], [6, -1, -1, -1]])
    refs = i32([2, 2, 1, 1, 1, 2, 2, 0])
    lens, need = [-1, 40, -1, 16], [0, 64, 64, 64]
    got = update(ada, lens, need, 0, 0, 16, table, refs, False)
    same(got, oracle.update_pages(lens, need, 0, 0, 16, table, refs))
    assert got[0].tolist() == [[-1] * 4, [0, 1, 3, 2], [-1] * 4, [6, 4, 5, 7]] and got[1].tolist() == [1, 1, 1, 1, 1, 1, 2, 1]
    assert got[2].tolist() == [0, 64, 0, 64]


def test_update_when_the_pool_is_empty(ada):  # noqa: F811
    table, refs = np.full((3, 4), -1, np.int32), i32([0, 1, 0])
    same(update(ada, [0, 0, 0], [20, 20, 70], 0, 0, 16, table, refs, False),
         (i32([[0, 2, -1, -1], [-1] * 4, [-1] * 4]), i32([1, 1, 1]), i32([20, 0, 0])))
    same(update(ada, [0, 3], [20, 20], 0, 0, 16, np.full((2, 4), -1, np.int32), i32([]), False),
         (np.full((2, 4), -1, np.int32), i32([]), i32([0, 3])))
    same(update(ada, [], [], 0, 0, 16, np.zeros((0, 4), np.int32), i32([3, 0]), False), (np.zeros((0, 4), np.int32), i32([3, 0]), i32([])))


def fork(ada, source, lens, ps, table, refs, in_place=False):  # noqa: F811
    import torch
    B, stride = len(source), table.shape[1]
    bt, rf = to_dev(table), to_dev(refs)
    out = [empty(B, stride), empty(B), rf if in_place else empty(len(refs)), empty(B), empty(B)]
    print("fork", len(table), "to", B, "stride", stride, "pages", len(refs), flush=True)
    ada.adaserve_fork_pages(source=to_dev(i32(source)), context_len=to_dev(i32(lens)), page_size=ps, block_table=bt, page_refs=rf,
                            new_block_table=out[0], new_context_len=out[1], new_page_refs=None if in_place else out[2],
                            copy_src=out[3], copy_dst=out[4], workspace=dev_workspace(ada, max(B, len(table)), len(refs)))
    torch.cuda.synchronize()
    assert np.array_equal(back(bt), table) and (in_place or np.array_equal(back(rf), refs))
    return [back(x) for x in out]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sources,rows,stride,pages,ps", [
    (1, 1, 1, 2, 16), (1, 8, 40, 60, 16), (8, 8, 20, 170, 16), (64, 64, 30, 2100, 16), (3, 1300, 4, 900, 16), (1100, 20, 3, 3400, 16),
    (5, 9, 300, 20000, 1), (4, 4, 9, 36, 5), (6, 30, 7, 44, 16), (512, 500, 12, 8192, 16), (500, 512, 12, 8193, 16),
    (513, 40, 11, 5000, 16), (40, 513, 11, 5000, 16),
])
def test_fork(ada, sources, rows, stride, pages, ps, in_place):  # noqa: F811
    rng = np.random.default_rng([sources, rows, stride])
    lens = rng.integers(-2, stride * ps + 3, sources)
    table, refs = tables(rng, sources, stride, pages, np.clip(lens, 0, stride * ps), ps, extra=0.02, spare=int(rng.integers(0, 3)))
    source = rng.integers(-1, sources + 1, rows)
    got = fork(ada, source, lens, ps, table, refs, in_place)
    same(got, oracle.fork_pages(source, lens, ps, table, refs))


def test_fork_to_nobody_and_from_nobody(ada):  # noqa: F811
    table, refs = i32([[0, 1], [2, -1]]), i32([1, 1, 1, 0])
    same(fork(ada, [], [20, 3], 16, table, refs), (np.zeros((0, 2), np.int32), i32([]), i32([0, 0, 0, 0]), i32([]), i32([])))
    same(fork(ada, [0, -1], [], 16, np.zeros((0, 2), np.int32), refs), (np.full((2, 2), -1), [0, 0], refs, [-1, -1], [-1, -1]))


def test_fork_takes_the_pages_that_it_frees(ada):  # noqa: F811
    """Beams: the last page of a beam that dies holds another one's copy, so a full pool is enough."""
    table, refs = i32([[0, 2], [1, 3], [5, 4]]), i32([1] * 6)
    got = fork(ada, [0, 0, 0], [20, 20, 20], 16, table, refs)
    assert got[0].tolist() == [[0, 2], [0, 1], [0, 3]] and got[2].tolist() == [3, 1, 1, 1, 0, 0]
    assert got[3].tolist() == [-1, 2, 2] and got[4].tolist() == [-1, 1, 3] and got[1].tolist() == [20, 20, 20]


def compact(ada, table, refs, in_place=False):  # noqa: F811
    import torch
    (B, stride), P = table.shape, len(refs)
    bt, rf = to_dev(table), to_dev(refs)
    out = [bt if in_place else empty(B, stride), rf if in_place else empty(P), empty(P), empty(P), empty(P), empty(2)]
    print("compact", B, stride, "pages", P, flush=True)
    ada.adaserve_compact_pages(block_table=bt, page_refs=rf, new_block_table=None if in_place else out[0],
                               new_page_refs=None if in_place else out[1], new_place=out[2], move_src=out[3], move_dst=out[4],
                               counts=out[5], workspace=dev_workspace(ada, B, P))
    torch.cuda.synchronize()
    assert in_place or (np.array_equal(back(bt), table) and np.array_equal(back(rf), refs))
    return [back(x) for x in out]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("used", [0.0, 0.03, 0.5, 0.97, 1.0])
@pytest.mark.parametrize("pages", [0, 1, 63, 64, 1024, 1025, 4096, 4097, 70001])
def test_compact(ada, pages, used, in_place):  # noqa: F811
    rng = np.random.default_rng([pages, int(used * 100)])
    refs = np.where(rng.random(pages) < used, rng.integers(1, 4, pages), -rng.integers(0, 2, pages)).astype(np.int32)
    table = rng.integers(-3, pages + 3, (5, 77)).astype(np.int32)
    same(compact(ada, table, refs, in_place), oracle.compact_pages(table, refs))


@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hkv,ps,d", [(1, 1, 8), (8, 16, 128), (3, 16, 64), (2, 5, 40), (16, 64, 128)])
def test_copy(ada, hkv, ps, d, dtype, layers):  # noqa: F811
    """Bit for bit, NaN patterns too; pairs that name no page are left out, and so are those behind the count."""
    import torch
    P = 12
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    bits = torch.int16 if dtype == "bf16" else torch.int32
    shape = (layers, P, hkv, ps, d) if layers > 1 else (P, hkv, ps, d)
    pools = [torch.randint(-30000, 30000, shape, dtype=bits, device="cuda") for _ in range(2)]
    src, dst = i32([3, 7, 3, -1, 4, P, 9, 5]), i32([0, 1, 2, 6, P, 8, 9, 10])
    for count in (None, 0, 2, 8, 100, -4):
        n = 8 if count is None else max(0, min(count, 8))
        expected = []
        for pool in pools:
            e = pool.clone()
            for a, b in zip(src[:n], dst[:n]):
                if 0 <= a < P and 0 <= b < P:
                    e[..., b, :, :, :] = pool[..., a, :, :, :]
            expected.append(e)
        got = [pool.clone() for pool in pools]
        print("copy", hkv, ps, d, dtype, layers, count, flush=True)
        ada.adaserve_copy_pages(src=to_dev(src), dst=to_dev(dst), count=None if count is None else to_dev(i32([count])),
                                k_pages=got[0].view(t), v_pages=got[1].view(t))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, expected))


def test_pages_from_a_graph(ada):  # noqa: F811
    """A captured update and fork, replayed as the tables change."""
    import torch
    rng = np.random.default_rng(11)
    B, stride, P, ps = 6, 12, 90, 16
    lens_host = rng.integers(0, 100, B)
    table_host, refs_host = tables(rng, B, stride, P, lens_host, ps)
    table_host = np.where(table_host >= P, -1, table_host).astype(np.int32)
    table, refs, lens, need = to_dev(table_host), to_dev(refs_host), to_dev(i32(lens_host)), to_dev(i32(lens_host + 1))
    source, cap = to_dev(i32(range(B))), empty(B)
    other, new_lens, src, dst = empty(B, stride), empty(B), empty(B), empty(B)
    ws = dev_workspace(ada, B, P)

    def step():
        ada.adaserve_update_pages(context_len=lens, need_len=need, window=50, sinks=4, page_size=ps, block_table=table,
                                  page_refs=refs, capacity=cap, workspace=ws)
        ada.adaserve_fork_pages(source=source, context_len=lens, page_size=ps, block_table=table, page_refs=refs,
                                new_block_table=other, new_context_len=new_lens, copy_src=src, copy_dst=dst, workspace=ws)
        table.copy_(other)
        lens.copy_(new_lens)

    start = [x.clone() for x in (table, refs, lens)]
    step()
    torch.cuda.synchronize()
    for x, y in zip((table, refs, lens), start):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    t, f, c = table_host, refs_host, i32(lens_host)
    for i in range(6):
        n = c + rng.integers(1, 20, B)
        n = np.minimum(n, stride * ps)
        s = rng.integers(0, B, B)
        need.copy_(to_dev(i32(n)))
        source.copy_(to_dev(i32(s)))
        graph.replay()
        torch.cuda.synchronize()
        t, f, capacity = oracle.update_pages(c, n, 50, 4, ps, t, f)
        t, c, f, a, b = oracle.fork_pages(s, c, ps, t, f)
        same([back(x) for x in (table, refs, lens, cap, src, dst)], [t, f, c, capacity, a, b])
        c = np.minimum(c + rng.integers(0, 9, B), (t >= 0).sum(1) * ps).astype(np.int32)
        lens.copy_(to_dev(c))
        torch.cuda.synchronize()
