"""The pages of the cache: calls at the ends of what is documented, against plain loops over the same tables."""
import numpy as np
import pytest

from oracle import window as oracle
from serving_inputs import to_dev
from test_gpu_pages import compact, fork, i32, same, update
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def test_no_rows_and_no_pages(ada):  # noqa: F811
    """Tables and pools of nothing, with a workspace of as many bytes as are asked for."""
    none = np.zeros((0, 4), np.int32)
    assert ada.adaserve_pages_workspace_bytes(0, 0) == 0
    same(update(ada, [], [], 0, 0, 16, none, i32([]), False), (none, i32([]), i32([])))
    same(fork(ada, [], [], 16, none, i32([])), (none, i32([]), i32([]), i32([]), i32([])))
    for in_place in (False, True):
        same(compact(ada, none, i32([]), in_place), oracle.compact_pages(none, i32([])))


@pytest.mark.parametrize("stride", [2 ** 63 - 1, -2 ** 63, 0])
def test_copies_of_one_layer_at_any_stride(ada, stride):  # noqa: F811
    import torch
    pools = [torch.randn(6, 2, 16, 64, device="cuda") for _ in range(2)]
    expected = [p.clone() for p in pools]
    for p in expected:
        p[4] = p[1]
    src, dst = to_dev(i32([1])), to_dev(i32([4]))
    print("copy, one layer, stride", stride, flush=True)
    status = ada.load_library().adaserve_copy_pages(1, src.data_ptr(), dst.data_ptr(), None, pools[0].data_ptr(), pools[1].data_ptr(),
                                                    1, stride, 6, 2, 16, 64, ada.ADASERVE_F32, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert status == 0 and all(torch.equal(x, y) for x, y in zip(pools, expected))


def test_most_rows_and_pages(ada):  # noqa: F811
    """65536 rows over 2^23 pages: every row takes pages, the last ones those behind all others."""
    rng = np.random.default_rng(2)
    B, P, stride, ps = 65536, 2 ** 23, 3, 16
    refs = (rng.random(P) < 0.98).astype(np.int32)
    table = np.full((B, stride), -1, np.int32)
    lens, need = np.zeros(B, int), rng.integers(0, 3 * ps + 1, B)
    got = update(ada, lens, need, 0, 0, ps, table, refs, False)
    entries = -(-need // ps)
    free = np.flatnonzero(refs == 0)
    wanted = np.arange(stride)[None, :] < entries[:, None]
    assert wanted.sum() < free.size
    table[wanted] = free[:wanted.sum()]
    refs[table[wanted]] = 1
    same(got, (table, refs, i32(need)))
    # and every row over to another one, in which the partly filled pages are copied
    source = rng.integers(0, B, B)
    new, lens, counts, src, dst = fork(ada, source, need, ps, table, refs)
    first = np.full(B, B)
    np.minimum.at(first, source, np.arange(B))
    is_first = first[source] == np.arange(B)
    whole = need[source] // ps
    old, row, inside = table[source], np.arange(B), np.minimum(whole, stride - 1)
    kept = np.where((np.arange(stride)[None, :] < whole[:, None]) | is_first[:, None], old, -1)
    takes = ~is_first & (need[source] % ps != 0)
    after = refs.copy()
    np.add.at(after, old[kept >= 0], 1)
    np.add.at(after, table[table >= 0], -1)
    free = np.flatnonzero(after <= 0)[:takes.sum()]
    kept[row[takes], whole[takes]] = free
    after[free] = 1
    same((new, lens, counts), (kept, i32(need[source]), after))
    same((src, dst), (np.where(takes, old[row, inside], -1), np.where(takes, kept[row, inside], -1)))
