"""Arguments of the pages' entry points at the ends of their types, on the host before any HIP call."""
import pytest

import paper_2501_12162_amd as ada
from test_abi_window import BAD, UNSUP, _compact, _copy, _fork, _update, at, lib  # noqa: F401  (a fixture)

INT64_MAX = 2 ** 63 - 1


@pytest.mark.parametrize("dtype", [ada.ADASERVE_BF16, ada.ADASERVE_F32])
@pytest.mark.parametrize("stride,code", [(2 ** 62, UNSUP), (2 ** 61, UNSUP), (INT64_MAX, UNSUP), (INT64_MAX - 15, UNSUP),
                                         (2 ** 47 + 16, UNSUP), (2 ** 47 - 1, BAD), (-1, BAD), (-INT64_MAX - 1, BAD)])
def test_layer_strides_beyond_any_pool(lib, stride, code, dtype):  # noqa: F811
    """Their bytes do not fit 64 bits: refused without a product that overflows."""
    assert _copy(lib, stride=stride, dtype=dtype) == code and lib.adaserve_last_error()


def test_nothing_to_copy_at_any_stride(lib):  # noqa: F811
    for stride in (INT64_MAX, -INT64_MAX - 1):
        assert _copy(lib, n=0, layers=1, stride=stride) == 0


def test_calls_of_nothing_take_no_workspace(lib):  # noqa: F811
    """No rows and no pages need 0 bytes, and a tensor of 0 bytes has no address."""
    assert lib.adaserve_pages_workspace_bytes(0, 0) == 0
    assert lib.adaserve_update_pages(0, None, None, 0, 0, 16, None, 4, None, 0, None, None, None, None, 0, None) == 0
    assert lib.adaserve_fork_pages(0, 0, None, None, 16, None, 4, None, 0, None, None, None, None, None, None, 0, None) == 0


def test_arrays_of_nothing_overlap_nothing(lib):  # noqa: F811
    """Tables of no entries whose addresses lie within other arrays: calls fail for what they lack, not for these."""
    inside = at(4) + 16
    assert _update(lib, bts=0, bt=inside, nbt=inside, cap=at(1)) == BAD and b"capacity overlaps context_len" in lib.adaserve_last_error()
    assert _fork(lib, bts=0, bt=inside, nbt=inside, cs=at(9)) == BAD and b"copy_dst overlaps copy_src" in lib.adaserve_last_error()
    assert _compact(lib, bts=0, bt=at(2) + 4, nbt=at(2) + 4, ms=at(7)) == BAD
    assert b"move_dst overlaps move_src" in lib.adaserve_last_error()
