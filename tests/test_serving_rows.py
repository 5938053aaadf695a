"""Which rows of queries, keys and values the serving operators' binding takes as they lie."""
import numpy as np
import pytest
import torch

import paper_2501_12162_amd as ada


@pytest.mark.parametrize("x,step", [
    (torch.empty(5, 2, 64), 128), (torch.empty(5, 6, 64)[:, 2:4], 384), (torch.empty(5, 6, 64)[:, 2:3], 384),
    (torch.empty(1, 5, 64).transpose(0, 1), 64),            # one head whose step is another axis's
    (torch.empty(2, 5, 64)[1:].transpose(0, 1), 64), (torch.empty(1, 2, 64), 128), (torch.empty(0, 2, 64), 128),
    (torch.empty(5, 1, 1), 1),
])
def test_dense_heads_are_taken(x, step):
    assert ada._rows(x, "x") == (x.data_ptr(), step)


@pytest.mark.parametrize("x", [
    torch.empty(5, 64, 2).transpose(1, 2), torch.empty(5, 1, 128)[:, :, ::2], torch.empty(2, 5, 64).transpose(0, 1),
    torch.empty(5, 4, 64)[:, ::2], torch.empty(5, 3, 1)[:, ::2],
])
def test_heads_apart_are_refused(x):
    with pytest.raises(ValueError):
        ada._rows(x, "x")


@pytest.mark.gpu
def test_append_of_one_transposed_head():
    """Keys and values of one head as [1, tokens, D] seen as [tokens, 1, D] equal the same rows dense."""
    torch.manual_seed(3)
    k, v = (torch.randn(1, 7, 64, device="cuda").transpose(0, 1) for _ in range(2))
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    got = []
    for a, b in ((k, v), (k.contiguous(), v.contiguous())):
        pools = [torch.zeros(2, 1, 16, 64, device="cuda") for _ in range(2)]
        new = i32([0])
        ada.adaserve_rope_append_kv(token_indptr=i32([0, 7]), prefix_len=i32([12]), k=a, v=b, inv_freq=torch.ones(32, device="cuda"),
                                    k_pages=pools[0], v_pages=pools[1], block_table=i32([[1, 0]]), new_prefix_len=new)
        torch.cuda.synchronize()
        assert new.tolist() == [19]
        got.append([p.cpu().numpy() for p in pools])
    assert all(np.array_equal(x, y) for x, y in zip(*got)) and got[0][1].any()
