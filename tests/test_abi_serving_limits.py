"""Sizes at the ends of what the serving operators take, on the host before any
HIP call: workspaces that do not hold what the kernels write, and counts whose
sums leave 32 bits or one launch."""
import numpy as np
import pytest

import paper_2501_12162_amd as ada
from test_abi_serving import BAD, FAKE, SIZE_MAX, UNSUP, WS, _append, _decode, _prompt, _sample, lib  # noqa: F401

INT_MAX = 2 ** 31 - 1


def test_prompt_workspace_query_of_the_most_rows(lib):  # noqa: F811
    """2^31 - 1 rows, some of them far before their request's keys, others far behind."""
    ip, ctx = np.asarray([0, INT_MAX - 1, INT_MAX], np.int32), np.asarray([0, 2 ** 23 - 1], np.int32)
    assert lib.adaserve_prompt_attn_workspace_bytes(2, ip.ctypes.data, ctx.ctypes.data, 1, 1, 128, 16, ada.ADASERVE_BF16) == 0


def test_rows_whose_span_leaves_the_address_space(lib):  # noqa: F811
    """Spans of 2^31 rows at the largest stride, whose byte count is beyond 64 bits: refused, not wrapped into a range that
    overlaps nothing (or something)."""
    far = 2 ** 40
    assert _append(lib, T=INT_MAX, qs=far) == UNSUP
    assert _append(lib, T=INT_MAX, ks=far, q=None, qo=None) == UNSUP
    assert _append(lib, T=INT_MAX, vs=far) == UNSUP
    assert _append(lib, T=2 ** 9, qs=far) == UNSUP          # 2^49 elements
    assert _prompt(lib, ip=[0, 2 ** 27, 2 ** 27], qs=far) == UNSUP
    assert _decode(lib, B=2 ** 24, qs=far) == UNSUP
    assert _sample(lib, rows=2 ** 20, stride=2 ** 62) == UNSUP


def test_calls_of_more_threads_than_a_launch_takes(lib):  # noqa: F811
    """HIP launches fewer than 2^32 threads: calls that would need more are refused before anything is enqueued."""
    dense = dict(qs=64, ks=64, vs=64, hq=1, hkv=1, d=64, rot=64, qo=0x7000000000, kp=0x8000000000, vp=0x9000000000,
                 q=0x1000000000, k=0x2000000000, v=0x3000000000)
    assert _append(lib, T=2 ** 24, **dense) == UNSUP                       # a workgroup of 256 per token
    assert _append(lib, B=2 ** 26, T=5, new=0x10000000000) == UNSUP        # and one per four requests' lengths
    many = 2 ** 20                                                         # requests of a token: a workgroup each per kv-head
    assert _prompt(lib, dtype=ada.ADASERVE_F32, ip=np.arange(many + 1), ctx=np.zeros(many), hq=16, hkv=16, d=64) == UNSUP
    assert _prompt(lib, ip=np.arange(many + 1), ctx=np.zeros(many), hq=16, hkv=16, d=64) == UNSUP
    assert _decode(lib, B=2 ** 24, hq=1, hkv=1, d=64, qs=64) == UNSUP      # a workgroup per request and kv-head
    for rows in (2 ** 22, 2 ** 25):                                        # a workgroup of 1024 per row
        assert _sample(lib, rows=rows, wsb=2 ** 60) == UNSUP
        assert lib.adaserve_sample_workspace_bytes(rows, 100, ada.ADASERVE_F32) == SIZE_MAX
    assert lib.adaserve_sample_workspace_bytes(2 ** 22 - 1, 100, ada.ADASERVE_F32) != SIZE_MAX
    assert lib.adaserve_decode_attn_workspace_bytes(2 ** 24, 32, 1, 1, 64, 16, ada.ADASERVE_F32) == SIZE_MAX


def _need_prompt(lib, ip, ctx):
    ip, ctx = np.asarray(ip, np.int32), np.asarray(ctx, np.int32)
    return lib.adaserve_prompt_attn_workspace_bytes(ctx.size, ip.ctypes.data, ctx.ctypes.data, 8, 2, 128, 16, ada.ADASERVE_BF16)


def _workspace_cases(lib):
    """Per entry point: its call with a workspace, the bytes it needs, and those of a smaller batch."""
    prompt = dict(ip=[0, 64], ctx=[8064], bts=504)
    yield (lambda **kw: _prompt(lib, **prompt, **kw), _need_prompt(lib, [0, 64], [8064]), _need_prompt(lib, [0, 64], [2000]))
    decode = lambda B, most: lib.adaserve_decode_attn_workspace_bytes(B, most, 8, 2, 128, 16, ada.ADASERVE_BF16)
    yield (lambda **kw: _decode(lib, B=3, most=4096, bts=256, **kw), decode(3, 4096), decode(3, 600))
    sample = lambda rows, vocab: lib.adaserve_sample_workspace_bytes(rows, vocab, ada.ADASERVE_F32)
    yield (lambda **kw: _sample(lib, rows=3, **kw), sample(3, 100), sample(2, 100))
    yield (lambda **kw: _sample(lib, rows=3, vocab=20000, stride=20000, **kw), sample(3, 20000), sample(3, 4000))


@pytest.mark.parametrize("which", range(4))
def test_workspaces_that_are_missing_too_small_or_misaligned(lib, which):  # noqa: F811
    call, need, smaller = list(_workspace_cases(lib))[which]
    assert 0 < smaller < need < SIZE_MAX
    at = FAKE * 256
    assert call(ws=None, wsb=need) == WS and lib.adaserve_last_error()
    assert call(ws=at, wsb=0) == WS
    assert call(ws=at, wsb=need - 1) == WS
    assert call(ws=at, wsb=smaller) == WS           # asked for a batch before this one
    assert call(ws=at + 16, wsb=need) == BAD
