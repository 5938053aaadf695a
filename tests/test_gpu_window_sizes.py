"""Attention over a window and sinks in batches that take the ways of large calls: several tiles per workgroup, wide fp32
tiles, split prefixes; and keys that are not a number."""
import numpy as np
import pytest

import window_calls as calls
import window_dense as dense
from paged_calls import starts
from serving_inputs import PS, typed
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

PROMPT_ROWS, RESIDENT = 256, 256     # rows of a bf16 prompt's tile, workgroups on the device


def tiles(new, group, rows):
    return sum(-(-n * group // rows) for n in new)


def run_and_check(ada, kind, dtype, d, hq, hkv, new, ctx, window, sinks, seed):  # noqa: F811
    rng = np.random.default_rng(seed)
    cache, trees, q = calls.case(rng, kind, dtype, d, hq, hkv, new, ctx, window, sinks)
    got = calls.run(ada, kind, dtype, cache, trees, q, new, ctx, d ** -0.5, window, sinks)
    calls.check(kind, dtype, got, dense.expected(kind, cache, trees, q, new, ctx, d ** -0.5, window, sinks), window + sinks + 300)


@pytest.mark.parametrize("window,sinks", [(300, 4), (77, 0), (640, 70)])
@pytest.mark.parametrize("before", ["none", "near", "far"])
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_more_tiles_than_workgroups(ada, d, before, window, sinks):  # noqa: F811
    """A workgroup's tiles follow each other, each with a window of its own: whole prompts, unequal cached lengths within
    the window (a workgroup per tile), and beyond it (several, in order)."""
    new = [1100, 1030, 1200, 1025, 1, 1100, 1290, 1111, 1040]
    hq, hkv = 16, 4
    first = {"none": [0] * 9, "near": [0, 9, window - 1, 40, 300, 200, 5, 130, 260],
             "far": [window + x for x in (0, 500, 13, 900, 47, 260, 128, 31, 700)]}[before]
    ctx = [n + b for n, b in zip(new, first)]
    code = ada.ADASERVE_BF16
    assert tiles(new, hq // hkv, PROMPT_ROWS) * hkv > 2 * RESIDENT
    assert ada.adaserve_window_prompt_attn_workspace_bytes(starts(new), np.asarray(ctx, np.int32), hq, hkv, d, PS, window, sinks, code) == 0
    run_and_check(ada, "prompt", "bf16", d, hq, hkv, new, ctx, window, sinks, [d, window, len(before)])


@pytest.mark.parametrize("window,sinks", [(300, 4), (50, 40)])
@pytest.mark.parametrize("cached", [0, 333])
@pytest.mark.parametrize("d", [64, 128])
def test_f32_prompts_of_wide_tiles(ada, d, cached, window, sinks):  # noqa: F811
    new, heads = [1100, 900, 1300, 850, 33], 16
    ctx = [n + cached * i for i, n in enumerate(new)]
    assert tiles(new, 1, 32) * heads >= 2048
    run_and_check(ada, "prompt", "f32", d, heads, heads, new, ctx, window, sinks, [d, window, cached])


@pytest.mark.parametrize("window,sinks", [(300, 4), (20, 0), (9, 33)])
@pytest.mark.parametrize("d", [64, 128])
def test_f32_trees_of_wide_tiles(ada, d, window, sinks):  # noqa: F811
    new, ctx, hq, hkv = [128, 100, 128, 77, 128, 128], [700, 3, 290, 1500, 0, 310], 16, 4
    assert tiles(new, hq // hkv, 32) * hkv >= RESIDENT
    run_and_check(ada, "tree", "f32", d, hq, hkv, new, ctx, window, sinks, [d, window])


@pytest.mark.parametrize("window,sinks", [(1500, 4), (2047, 100)])
@pytest.mark.parametrize("d", [64, 128])
def test_trees_of_split_prefixes_are_rounded_once(ada, d, window, sinks):  # noqa: F811
    """The chunks' outputs are fp32: the means are as near as those of one piece."""
    rng = np.random.default_rng([d, window])
    new, ctx, hq, hkv = [9, 20, 64], [900, 2100, 5000], 8, 2
    cache, trees, q = calls.case(rng, "tree", "bf16", d, hq, hkv, new, ctx, window, sinks, whole=True)
    need = ada.adaserve_window_tree_attn_workspace_bytes(trees.indptr, np.asarray(ctx, np.int32), hq, hkv, d, PS, window, sinks,
                                                         ada.ADASERVE_BF16)
    assert need > 0
    got = calls.run(ada, "tree", "bf16", cache, trees, q, new, ctx, 0.09, window, sinks)
    out, size, _ = dense.expected("tree", cache, trees, q, new, ctx, 0.09, window, sinks)
    over = float((np.abs(got - out) - dense.split_mean_bound(out, size)).max())
    assert over <= 0, over


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("column", [False, True])
def test_prompts_of_a_sink_that_is_not_a_number(ada, dtype, column):  # noqa: F811
    """All rows behind it see it: they are NaN, in its column alone where only a value there is."""
    rng = np.random.default_rng(4)
    n, window, sinks, d = 900, 200, 4, 128
    cache, _, q = calls.case(rng, "prompt", dtype, d, 4, 2, [n], [n], window, sinks)
    clean = dense.expected("prompt", cache, None, q, [n], [n], 0.09, window, sinks)
    nan = typed(np.full(1, np.nan, np.float32), dtype)[0]
    page = cache.table[0, 0]
    if column:
        cache.v[page, :, 2, 17] = nan
    else:
        cache.k[page, :, 2], cache.v[page, :, 2] = nan, nan
    got = calls.run(ada, "prompt", dtype, cache, None, q, [n], [n], 0.09, window, sinks)
    hit = np.zeros(d, bool)
    hit[17 if column else slice(None)] = True
    assert np.isnan(got[2:][..., hit]).all()
    calls.check("prompt", dtype, got[:2], tuple(x[:2] for x in clean), 300)
    if column:
        got[2:, :, 17] = clean[0][2:, :, 17]
        calls.check("prompt", dtype, got, clean, 300)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("at", [1, 2100, 2399])
def test_a_token_of_a_key_that_is_not_a_number(ada, dtype, at):  # noqa: F811
    """A sink, a key of the window, the token's own: its request is NaN, the ones beside it are as without it."""
    rng = np.random.default_rng(at)
    ctx, window, sinks = [300, 2400, 1700], 1000, 4
    cache, _, q = calls.case(rng, "decode", dtype, 128, 8, 2, None, ctx, window, sinks)
    clean = calls.expected("decode", cache, None, q, None, ctx, 0.09, window, sinks)
    cache.k[cache.table[1, at // PS], :, at % PS] = typed(np.full(1, np.nan, np.float32), dtype)[0]
    got = calls.run(ada, "decode", dtype, cache, None, q, None, ctx, 0.09, window, sinks)
    assert np.isnan(got[1]).all()
    calls.check("decode", dtype, got[[0, 2]], tuple(x[[0, 2]] for x in clean), 1100)
