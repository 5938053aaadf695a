"""GPU parity of adaserve_sample with the oracle: the same token in every row."""
import numpy as np
import pytest

from oracle import serving
from serving_inputs import back, to_dev, typed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ada():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2501_12162_amd as ada
    ada.load_library()
    return ada


def draw(ada, logits, vocab, u, workspace=None, out=None, check=True, **par):
    """`logits` [rows, width] typed host rows; par: host arrays of the parameters given."""
    import torch
    rows = len(logits)
    x = to_dev(logits)
    need = ada.adaserve_sample_workspace_bytes(rows, vocab, ada.ADASERVE_F32 if logits.dtype == np.float32 else ada.ADASERVE_BF16)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    out = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    kinds = {"temperature": np.float32, "top_k": np.int32, "top_p": np.float32, "min_p": np.float32}
    par = {k: np.asarray(v, kinds[k]) for k, v in par.items()}
    print("sample rows", rows, "vocab", vocab, "width", logits.shape[1], "workspace", need, flush=True)
    ada.adaserve_sample(logits=x, vocab=vocab, u=to_dev(np.asarray(u, np.float32)), out_token=out, workspace=ws,
                        **{k: to_dev(v) for k, v in par.items()})
    torch.cuda.synchronize()
    got = back(out)
    if check:
        ref = serving.sample(logits, vocab, u=np.asarray(u, np.float32), **par)
        assert got.tolist() == ref.tolist(), [(i, a, b) for i, (a, b) in enumerate(zip(got, ref)) if a != b]
    return got


def parameters(rng, rows):
    """Every combination of filters, some of them off."""
    return dict(temperature=np.where(rng.random(rows) < 0.1, 0, rng.uniform(0.3, 2.0, rows)),
                top_k=np.where(rng.random(rows) < 0.4, 0, rng.integers(1, 200, rows)),
                top_p=np.where(rng.random(rows) < 0.3, 1.0, rng.uniform(0.05, 1.0, rows)),
                min_p=np.where(rng.random(rows) < 0.5, 0.0, rng.uniform(0, 0.2, rows)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,pad", [(1, 0), (2, 3), (7, 0), (63, 2), (64, 0), (65, 0), (1000, 1), (1024, 0), (4097, 0),
                                       (16384, 8), (16385, 0), (50257, 0), (128256, 5)])
def test_sample_vocabularies(ada, dtype, vocab, pad):
    rng = np.random.default_rng(vocab)
    rows = 24 if vocab < 5000 else 12
    x = typed(rng.standard_normal((rows, vocab + pad)) * 3, dtype)
    if pad:
        x[:, vocab:] = typed(np.array([np.nan]), dtype)
    draw(ada, x, vocab, rng.random(rows), **parameters(rng, rows))
    draw(ada, x, vocab, rng.random(rows))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spread", [0.0, 0.01, 0.5, 4.0, 40.0])
def test_sample_spreads(ada, dtype, spread):
    """From all tokens equal (one tie of the whole row) to one token with all the mass."""
    rng = np.random.default_rng(int(spread * 100))
    rows, v = 40, 3000
    x = typed(rng.standard_normal((rows, v)) * spread, dtype)
    draw(ada, x, v, rng.random(rows), **parameters(rng, rows))
    draw(ada, x, v, rng.random(rows), top_k=[1, 2, 3, 2999] * 10, temperature=[5.0] * rows)
    draw(ada, x, v, rng.random(rows), top_p=np.linspace(0.01, 0.999, rows))


def test_sample_large_ties(ada):
    """Rows of few distinct values, in vocabularies whose ties fill more than any list kept of them."""
    rng = np.random.default_rng(4)
    rows, v = 12, 128256
    x = rng.integers(0, 3, (rows, v)).astype(np.float32)
    x[:3] = 1.5
    for dtype in ("bf16", "f32"):
        draw(ada, typed(x, dtype), v, rng.random(rows), top_k=[0, 5, 70000, 128255] * 3)
        draw(ada, typed(x, dtype), v, rng.random(rows), top_p=[0.1, 0.5, 0.9, 0.9999] * 3)
        draw(ada, typed(x, dtype), v, rng.random(rows), top_k=[100000] * rows, top_p=[0.7] * rows, min_p=[0.3] * rows)


def test_sample_signed_zeros_tie(ada):
    x = np.zeros((6, 70), np.float32)
    x[:, ::2] = -0.0
    for dtype in ("bf16", "f32"):
        draw(ada, typed(x, dtype), 70, [0, 0.3, 0.5, 0.7, 0.9, 0.99], top_k=[3] * 6)
        draw(ada, typed(x, dtype), 70, [0, 0.3, 0.5, 0.7, 0.9, 0.99])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_border_values(ada, dtype):
    """Masks of -inf and of the type's lowest value, rows without a token, NaN
    and +inf; uniforms 0, next below 1, 1 and beyond; filters at and past their ends."""
    rng = np.random.default_rng(6)
    v = 400
    base = rng.standard_normal((16, v)) * 2
    low = -3.3895e38
    base[1, :] = -np.inf
    base[2, :-1] = -np.inf
    base[3, ::2] = low
    base[4, :] = low
    base[5, 17] = np.nan
    base[6, 399] = np.inf
    base[7, 0] = -np.nan
    base[8, 5:] = -np.inf
    base[9, :] = 3.3e38
    x = typed(base, dtype)
    just = np.nextafter(np.float32(1), np.float32(0))
    for u in (0.0, 0.5, just, 1.0, 2.0, -1.0, np.nan):
        draw(ada, x, v, np.full(16, u))
        draw(ada, x, v, np.full(16, u), top_k=np.full(16, 3), top_p=np.full(16, 0.9), min_p=np.full(16, 0.01))
    u = rng.random(16)
    for k in (-5, 0, 1, 399, 400, 401, 2 ** 31 - 1, -2 ** 31):
        draw(ada, x, v, u, top_k=np.full(16, k))
    for p in (-1.0, 0.0, 1e-30, 0.5, just, 1.0, 5.0, np.inf, -np.inf, np.nan):
        draw(ada, x, v, u, top_p=np.full(16, p))
        draw(ada, x, v, u, min_p=np.full(16, p))
    for t in (0.0, -0.0, 1e-30, 0.01, 1e30, 3e38, np.inf, -1.0, np.nan):
        draw(ada, x, v, u, temperature=np.full(16, t))
        draw(ada, x, v, u, temperature=np.full(16, t), top_k=np.full(16, 50), top_p=np.full(16, 0.9))


def test_sample_rows_apart(ada):
    """Rows inside a wider array, at every alignment of the element."""
    import torch
    rng = np.random.default_rng(7)
    for dtype in ("bf16", "f32"):
        for shift in range(1, 9):
            whole = typed(rng.standard_normal((9, 2031 + shift)) * 3, dtype)
            x = to_dev(whole)[:, shift:shift + 2020]
            u = rng.random(9).astype(np.float32)
            out = torch.empty(9, dtype=torch.int32, device="cuda")
            need = ada.adaserve_sample_workspace_bytes(9, 2019, ada.ADASERVE_BF16 if dtype == "bf16" else ada.ADASERVE_F32)
            ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
            p = to_dev(np.full(9, 0.8, np.float32))
            ada.adaserve_sample(logits=x, vocab=2019, u=to_dev(u), out_token=out, top_p=p, workspace=ws)
            torch.cuda.synchronize()
            ref = serving.sample(whole[:, shift:], 2019, top_p=np.full(9, 0.8, np.float32), u=u)
            assert back(out).tolist() == ref.tolist(), (dtype, shift)


@pytest.mark.parametrize("seed", range(6))
def test_sample_drawn(ada, seed):
    rng = np.random.default_rng(50 + seed)
    v = int(rng.choice([300, 5000, 32000, 151936]))
    rows = int(rng.integers(1, 6 if v > 10000 else 70))
    x = typed(rng.standard_normal((rows, v)) * float(rng.choice([0.3, 2, 8])), str(rng.choice(["bf16", "f32"])))
    draw(ada, x, v, rng.random(rows), **parameters(rng, rows))


def test_sample_largest_vocabulary(ada):
    rng = np.random.default_rng(8)
    v = 1 << 20
    x = typed(rng.standard_normal((3, v)), "bf16")
    draw(ada, x, v, rng.random(3), top_k=[0, 1000, 0], top_p=[1.0, 0.5, 0.95])


def test_sample_replayed_from_a_graph(ada):
    """Replays with new logits, parameters and uniforms in place, an eager call
    of another batch in its own workspace between them."""
    import torch
    rng = np.random.default_rng(12)
    rows, v = 6, 20000
    x = to_dev(typed(rng.standard_normal((rows, v)), "bf16"))
    t, p, m, u = (to_dev(np.ones(rows, np.float32)) for _ in range(4))
    k = to_dev(np.zeros(rows, np.int32))
    out = torch.empty(rows, dtype=torch.int32, device="cuda")
    need = ada.adaserve_sample_workspace_bytes(rows, v, ada.ADASERVE_BF16)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")

    def call():
        ada.adaserve_sample(logits=x, vocab=v, u=u, out_token=out, temperature=t, top_k=k, top_p=p, min_p=m, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for rep in range(5):
        host = typed(rng.standard_normal((rows, v)) * (1 + rep), "bf16")
        par = parameters(rng, rows)
        uu = rng.random(rows).astype(np.float32)
        x.copy_(to_dev(host))
        for dev, name in ((t, "temperature"), (k, "top_k"), (p, "top_p"), (m, "min_p")):
            dev.copy_(torch.as_tensor(np.asarray(par[name], np.int32 if dev is k else np.float32)))
        u.copy_(torch.as_tensor(uu))
        out.fill_(-7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        par = {n: np.asarray(a, np.int32 if n == "top_k" else np.float32) for n, a in par.items()}
        assert back(out).tolist() == serving.sample(host, v, u=uu, **par).tolist(), rep
        draw(ada, typed(rng.standard_normal((3, 4000)), "f32"), 4000, rng.random(3))


def test_sample_rows_beyond_4_gib(ada):
    """Rows 2^28 fp32 elements apart: the last begins 9 GiB after the first."""
    import torch
    rng = np.random.default_rng(23)
    rows, vocab, step = 10, 5000, 2 ** 28
    x = typed(rng.standard_normal((rows, vocab)) * 3, "f32")
    far = torch.empty((rows - 1) * step + vocab, device="cuda").as_strided((rows, vocab), (step, 1))
    far.copy_(to_dev(x))
    u = rng.random(rows).astype(np.float32)
    out = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    ws = torch.empty(ada.adaserve_sample_workspace_bytes(rows, vocab, ada.ADASERVE_F32), dtype=torch.uint8, device="cuda")
    print("sample rows far apart", flush=True)
    ada.adaserve_sample(logits=far, vocab=vocab, u=to_dev(u), out_token=out, workspace=ws)
    torch.cuda.synchronize()
    assert back(out).tolist() == serving.sample(x, vocab, u=u).tolist()
