"""Prompt and single-token attention on caches where every key shows: means over
whole numbers, and queries that point at one key beside an end of something."""
import numpy as np
import pytest

from marked_caches import counted, mean_bound, means, pointed
from oracle import serving
from paged_calls import check, run_decode, run_prompt, starts
from serving_inputs import PS, Cache, typed
from test_gpu_paged_attention import HEADS, ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


def exactly(got, right, dtype):
    assert np.isfinite(got).all()
    err, b = np.abs(got - right), mean_bound(dtype, right) + 1e-30
    assert (err <= b).all(), (float((err / b).max()), int((err > b).sum()))


def decode_means(ada, ctx, dtype, hq=8, hkv=2, d=128, most=None):  # noqa: F811
    rng = np.random.default_rng(sum(ctx) % 2 ** 31)
    c = counted(rng, ctx, hkv, d, dtype)
    if most is not None:
        extra = -(-most // PS) - c.table.shape[1]
        c.table = np.concatenate([c.table, np.full((len(ctx), max(extra, 0)), -1, np.int32)], 1)
    got = run_decode(ada, typed(np.zeros((len(ctx), hq, d)), dtype), ctx, c, dtype, d ** -0.5, most=most)
    exactly(got, means(c, [1] * len(ctx), ctx, hq), dtype)


@DTYPES
@pytest.mark.parametrize("ctx", [[1, 2, 15, 16, 17, 31, 32, 33, 0], [4097, 1, 300], [9000], [20000, 0, 0, 31, 128], [2047, 2048, 2049] * 7,
                                 [513] * 40 + [0, 7000], [131072], [127, 128, 129, 0] * 260])
def test_decode_means(ada, dtype, ctx):  # noqa: F811
    decode_means(ada, ctx, dtype)


@DTYPES
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", HEADS + [(64, 8)])
def test_decode_means_heads(ada, dtype, d, hq, hkv):  # noqa: F811
    decode_means(ada, [5000, 33, 0, 700], dtype, hq, hkv, d)
    decode_means(ada, [300, 41, 0, 999, 17], dtype, hq, hkv, d, most=40000)


@DTYPES
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("ctx", [[4097, 1, 300], [20000, 129], [33] * 30 + [2048]])
def test_decode_pointed(ada, dtype, d, ctx):  # noqa: F811
    new = [1] * len(ctx)
    c, q = pointed(np.random.default_rng(sum(ctx)), new, ctx, 16, 4, d, dtype)
    check("decode", run_decode(ada, q, ctx, c, dtype, d ** -0.5), q, new, ctx, c, dtype, d ** -0.5)


@DTYPES
@pytest.mark.parametrize("ctx", [[17, 40, 3], [129, 300, 1500], [700] * 3])
def test_decode_weights(ada, dtype, ctx):  # noqa: F811
    """Ordinary queries, at the bound of weights of 16 bits."""
    rng = np.random.default_rng(sum(ctx))
    new = [1] * len(ctx)
    c = Cache(rng, ctx, 2, 128, dtype)
    q = typed(rng.standard_normal((len(ctx), 8, 128)), dtype)
    check("decode", run_decode(ada, q, ctx, c, dtype, 128 ** -0.5), q, new, ctx, c, dtype, 128 ** -0.5)


# (new, ctx, hq, hkv, what of it is split in bf16); the last three have tiles for the persistent grid, for it with keys
# before the rows, and more requests than the table of a launch takes
LISTS = [
    ([1, 2, 31, 32, 33, 0, 5], [1, 17, 31, 40, 33, 3, 2], 8, 2, None), ([300, 257], [300, 1000], 7, 1, None),
    ([70], [2049], 8, 2, True), ([257], [6500], 4, 2, True), ([1], [8000], 32, 2, True), ([2100], [4250], 16, 4, False),
    ([1100, 1030, 1200, 1025, 1, 1100, 1290, 1111, 1040], [1100, 1030, 1200, 1025, 1, 1100, 1290, 1111, 1040], 16, 4, False),
    ([2003, 2020, 2016, 1999], [2103, 2120, 2116, 2099], 32, 8, False), ([40] * 150 + [7] * 9, [50] * 150 + [7] * 9, 16, 16, False),
]
LIST = pytest.mark.parametrize("new,ctx,hq,hkv,split", LISTS)


@DTYPES
@pytest.mark.parametrize("d", [64, 128])
@LIST
def test_prompt_means(ada, dtype, d, new, ctx, hq, hkv, split):  # noqa: F811
    c = counted(np.random.default_rng(sum(ctx)), ctx, hkv, d, dtype)
    q = typed(np.zeros((sum(new), hq, d)), dtype)
    got = run_prompt(ada, q, new, ctx, c, dtype, d ** -0.5, split=split if dtype == "bf16" else False, pad=2)
    exactly(got, means(c, new, ctx, hq), dtype)


@DTYPES
@pytest.mark.parametrize("d", [64, 128])
@LIST
def test_prompt_pointed(ada, dtype, d, new, ctx, hq, hkv, split):  # noqa: F811
    c, q = pointed(np.random.default_rng(sum(ctx) + 1), new, ctx, hq, hkv, d, dtype)
    got = run_prompt(ada, q, new, ctx, c, dtype, d ** -0.5, split=split if dtype == "bf16" else False)
    check("prompt", got, q, new, ctx, c, dtype, d ** -0.5)


# ---- fp32 tiles of 32 rows (from 2048 of them on) ----

WIDE = [([1500, 1400, 1300, 1], 16, 16), ([700, 33, 650], 64, 32), ([15] * 140, 16, 16)]


def tiles(new, hq, hkv, rows=32):
    return sum(-(-n * (hq // hkv) // rows) for n in new) * hkv


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("before", [0, 100])
@pytest.mark.parametrize("new,hq,hkv", WIDE)
def test_f32_wide_tiles(ada, d, before, new, hq, hkv):  # noqa: F811
    assert tiles(new, hq, hkv) >= 2048
    rng = np.random.default_rng(d + before + len(new))
    ctx = [n + before for n in new]
    c = Cache(rng, ctx, hkv, d, "f32")
    q = typed(rng.standard_normal((sum(new), hq, d)), "f32")
    got = run_prompt(ada, q, new, ctx, c, "f32", d ** -0.5, pad=3)
    check("prompt", got, q, new, ctx, c, "f32", d ** -0.5)


@pytest.mark.parametrize("d", [64, 128])
def test_f32_wide_tiles_without_pages_or_keys(ada, d):  # noqa: F811
    """Pages outside the pool, fewer keys than rows, and no key at all."""
    new, ctx, hq, hkv = [1500, 1300, 40, 1300, 3], [1500, 1290, 0, 1400, 3], 16, 16
    assert tiles(new, hq, hkv) >= 2048
    rng = np.random.default_rng(d)
    c = Cache(rng, ctx, hkv, d, "f32")
    for r, e in ((0, 0), (0, 40), (0, 93), (1, 5), (1, 80), (3, 64), (3, 63), (4, 0)):
        c.table[r, e] = -1 if e % 2 else c.pages
    q = typed(rng.standard_normal((sum(new), hq, d)), "f32")
    got = run_prompt(ada, q, new, ctx, c, "f32", d ** -0.5)
    check("prompt", got, q, new, ctx, c, "f32", d ** -0.5)
    assert not got[1500:1510].any() and not got[2800:2840].any() and not got[-3:].any()


def hide(c, ctx, rows, bad, dtype):
    """The last `rows` keys and values of every request become `bad`."""
    for r, n in enumerate(ctx):
        for t in range(max(n - rows, 0), n):
            for pool in (c.k, c.v):
                pool[c.table[r, t // PS], :, t % PS] = typed(np.full(pool.shape[3], bad), dtype)


def seen_apart(got, q, new, ctx, rows, c, dtype, scale):
    """`got` of the rows that see none of the last `rows` keys of their requests, against the oracle on the rest."""
    first = starts(new)
    keep = np.concatenate([np.arange(a, a + max(n - rows, 0)) for a, n in zip(first, new)]).astype(int)
    check("prompt", got[keep], q[keep], [max(n - rows, 0) for n in new], [max(x - rows, 0) for x in ctx], c, dtype, scale)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan, 3.3e38])
@pytest.mark.parametrize("d", [64, 128])
def test_f32_wide_tiles_hidden_values(ada, d, bad):  # noqa: F811
    new, hq, hkv = [1500, 1400, 1300, 25], 16, 16
    assert tiles(new, hq, hkv) >= 2048
    ctx = [1500, 1450, 1300, 60]
    rng = np.random.default_rng(7)
    c = Cache(rng, ctx, hkv, d, "f32")
    hide(c, ctx, 20, bad, "f32")
    q = typed(rng.standard_normal((sum(new), hq, d)), "f32")
    seen_apart(run_prompt(ada, q, new, ctx, c, "f32", d ** -0.5), q, new, ctx, 20, c, "f32", d ** -0.5)


# ---- bf16 tiles that are done again, between others of the same workgroup ----

GRID = [1100, 1030, 1200, 1025, 1, 1100, 1290, 1111, 1040]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("every", [1, 2, 3])
def test_tiles_done_again_in_a_persistent_grid(ada, d, every):  # noqa: F811
    """Steep scores in every request, every second or every third: sums beyond 2^64 of the first keys' weights."""
    hq, hkv = 16, 4
    assert tiles(GRID, hq, hkv, 256) > 256
    rng = np.random.default_rng(d + every)
    c = Cache(rng, GRID, hkv, d, "bf16")
    k = serving.widen(c.k)
    for r, row in enumerate(c.table):
        if r % every == 0:
            for e, p in enumerate(row):
                if p >= 0:
                    k[p] *= (1 + e % 7 + (e > 40) * 9) * (-1) ** e
    c.k = typed(k, "bf16")
    q = typed(rng.standard_normal((sum(GRID), hq, d)), "bf16")
    got = run_prompt(ada, q, GRID, GRID, c, "bf16", d ** -0.5 * 8, split=False)
    check("prompt", got, q, GRID, GRID, c, "bf16", d ** -0.5 * 8)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [np.inf, np.nan, 3.3e38])
def test_hidden_values_in_a_persistent_grid(ada, d, bad):  # noqa: F811
    hq, hkv, rows = 16, 4, 20
    rng = np.random.default_rng(d)
    c = Cache(rng, GRID, hkv, d, "bf16")
    hide(c, GRID, rows, bad, "bf16")
    q = typed(rng.standard_normal((sum(GRID), hq, d)), "bf16")
    seen_apart(run_prompt(ada, q, GRID, GRID, c, "bf16", d ** -0.5, split=False), q, GRID, GRID, rows, c, "bf16", d ** -0.5)


def test_large_values_in_a_persistent_grid(ada):  # noqa: F811
    """The test of products beyond fp32 between tiles without any."""
    from test_gpu_attention_ranges import rising
    hq, hkv, d = 16, 4, 128
    rng = np.random.default_rng(1)
    c, q = rising(rng, GRID, GRID, hq, hkv, d, "bf16", 36.0, 2.0 ** 70, True)
    for r in range(0, len(GRID), 2):
        for p in c.table[r][c.table[r] >= 0]:
            c.v[p] = typed(rng.standard_normal(c.v[p].shape), "bf16")
    got = run_prompt(ada, q, GRID, GRID, c, "bf16", d ** -0.5, split=False)
    check("prompt", got, q, GRID, GRID, c, "bf16", d ** -0.5)
