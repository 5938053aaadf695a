"""Pins of the serving operators' oracle (oracle/serving.py): independent
routines, brute force and hand-worked values."""
import numpy as np
import pytest
import torch

from oracle import serving


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_is_a_complex_rotation(interleaved):
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 3, 16)), np.array([0, 1, 7, 1000, 8388607])
    inv = (10000.0 ** (-np.arange(6) / 6)).astype(np.float32)
    y = serving.rope(x, pos, inv, interleaved)
    pair = x[..., :12].reshape(5, 3, 6, 2) if interleaved else np.stack([x[..., :6], x[..., 6:12]], -1)
    z = (pair[..., 0] + 1j * pair[..., 1]) * np.exp(1j * pos[:, None] * inv.astype(np.float64))[:, None]
    got = y[..., :12].reshape(5, 3, 6, 2) if interleaved else np.stack([y[..., :6], y[..., 6:12]], -1)
    assert np.abs(got[..., 0] + 1j * got[..., 1] - z).max() < 1e-12
    assert np.array_equal(y[..., 12:], x[..., 12:]) and np.array_equal(y[0], x[0])   # unrotated part; position 0
    # scores depend on the distance of positions alone
    a, b = rng.standard_normal((2, 1, 1, 12))
    dot = [float((serving.rope(a, [p + 5], inv) * serving.rope(b, [p], inv)).sum()) for p in (0, 3, 900)]
    assert max(dot) - min(dot) < 1e-9


def test_append_places_by_hand():
    table = np.array([[4, 1, -1], [9, 2, 3], [0, 5, 6]])
    req, place, page, new = serving.append_places([0, 3, 3, 6], [3, 8, -2], table, 8, 4, 8)
    assert req.tolist() == [0, 0, 0, 2, 2, 2, -1, -1]
    assert place[:6].tolist() == [3, 4, 5, -2, -1, 0]
    assert page.tolist() == [4, 1, 1, -1, -1, -1, -1, -1] and new.tolist() == [6, 8, -2]
    _, _, page, new = serving.append_places([0, 6], [3], np.array([[4, -1, 7]]), 8, 4, 6)
    assert page.tolist() == [4, -1, -1, -1, -1, 7] and new.tolist() == [4]   # a hole ends the length


@pytest.mark.parametrize("n,c", [(1, 1), (5, 5), (4, 9), (7, 3), (3, 0), (1, 40)])
def test_paged_attention_against_a_library_routine(n, c):
    rng = np.random.default_rng(n * 100 + c)
    Hq, Hkv, D, ps = 4, 2, 8, 4
    pages = -(-c // ps)
    table = np.concatenate([rng.permutation(pages + 2)[:pages], [-1]])[None]
    kp, vp = rng.standard_normal((2, pages + 2, Hkv, ps, D))
    q = rng.standard_normal((n, Hq, D))
    out, size, _ = serving.paged_attention(q, [0, n], kp, vp, table, [c], 0.3)
    assert (size >= np.abs(out) - 1e-12).all()
    hidden = max(n - c, 0)
    assert not out[:hidden].any()
    if n > hidden:
        flat = lambda pool: torch.tensor(np.concatenate([pool[p] for p in table[0][:pages]], 1)[:, :c])
        k, v = (flat(x).repeat_interleave(2, 0) for x in (kp, vp))
        mask = torch.arange(c)[None] <= torch.arange(c - n, c)[:, None]
        ref = torch.nn.functional.scaled_dot_product_attention(torch.tensor(q).transpose(0, 1), k, v, mask, scale=0.3)
        assert np.abs(ref.transpose(0, 1).numpy()[hidden:] - out[hidden:]).max() < 1e-12


def test_sample_by_hand():
    x = np.log([4.0, 1.0, 2.0, 1.0])          # probabilities 1/2, 1/8, 1/4, 1/8
    draw = lambda u, t=1.0, k=0, p=1.0, m=0.0: serving.sample_row(x, t, k, p, m, u)
    assert [draw(u) for u in (0.0, 0.49, 0.51, 0.62, 0.63, 0.87, 0.88, 1.0)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [draw(u, k=2) for u in (0.0, 0.66, 0.67, 0.99)] == [0, 0, 2, 2]
    assert [draw(u, k=3) for u in (0.56, 0.58, 0.7, 0.72)] == [0, 1, 1, 2]        # the tie goes to index 1
    assert [draw(u, p=0.4) for u in (0.0, 0.99)] == [0, 0]
    assert [draw(u, p=0.6) for u in (0.66, 0.68)] == [0, 2]
    assert [draw(u, p=0.8) for u in (0.56, 0.58, 0.7, 0.72)] == [0, 1, 1, 2]
    assert [draw(u, k=2, p=0.66) for u in (0.5, 0.99)] == [0, 0]                  # 2/3 of the two: the first suffices
    assert [draw(u, m=0.3) for u in (0.66, 0.68)] == [0, 2]
    assert [draw(u, t=0.5) for u in (0.72, 0.73, 0.78)] == [0, 1, 2]              # 16 : 1 : 4 : 1
    assert draw(0.9, t=0.0) == 0 and draw(0.9, m=2.0) == 0 and draw(0.9, p=-1.0) == 0
    assert serving.sample_row(np.array([0.0, -0.0, 0.0]), 1.0, 1, 1.0, 0.0, 0.9) == 0
    assert serving.sample_row([1.0, np.nan], 1, 0, 1, 0, 0.5) == -1
    assert serving.sample_row([1.0, np.inf], 1, 0, 1, 0, 0.5) == -1
    assert serving.sample_row([-np.inf, -np.inf], 1, 0, 1, 0, 0.5) == -1
    assert serving.sample_row([-np.inf, -3e38], 1, 0, 1, 0, 0.5) == 1
    for bad in ((-1.0, 1.0, 0.0, 0.5), (np.nan, 1.0, 0.0, 0.5), (np.inf, 1.0, 0.0, 0.5), (1.0, np.nan, 0.0, 0.5),
                (1.0, 1.0, np.nan, 0.5), (1.0, 1.0, 0.0, np.nan)):
        assert serving.sample_row(x, bad[0], 0, *bad[1:]) == -1


@pytest.mark.parametrize("t,k,p,m", [(1.0, 0, 1.0, 0.0), (0.7, 5, 1.0, 0.0), (1.3, 0, 0.8, 0.0), (1.0, 7, 0.9, 0.05)])
def test_sample_follows_the_filtered_distribution(t, k, p, m):
    """Tokens at evenly spread uniforms come in the shares of the distribution
    that is filtered step by step on probabilities."""
    x = np.random.default_rng(3).standard_normal(12) * 2
    prob = np.exp(x / t) / np.exp(x / t).sum()
    order = np.argsort(-prob)[:k or None]
    kept = prob[order] / prob[order].sum()
    order = order[np.cumsum(kept) - kept < p]
    order = order[prob[order] >= m * prob.max()]
    share = np.zeros(12)
    share[order] = prob[order] / prob[order].sum()
    n = 4000
    got = np.bincount([serving.sample_row(x, t, k, p, m, (i + 0.5) / n) for i in range(n)], minlength=12) / n
    assert np.abs(got - share).max() <= 1.0 / n + 1e-9
