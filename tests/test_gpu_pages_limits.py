"""The pages of the cache: calls at the ends of what is documented, against plain loops over the same tables."""
import numpy as np
import pytest

from oracle import window as oracle
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
