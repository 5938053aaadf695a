"""Which tensors the pages' and the window attentions' entry points take: nothing is launched."""
import numpy as np
import pytest
import torch

import paper_2501_12162_amd as ada


class Fake:
    """What the binding asks of a tensor, on a device of choice."""

    def __init__(self, *shape, device=0, dtype=torch.int32, contiguous=True):
        self.shape, self.device_index, self.dtype, self.contiguous = torch.Size(shape), device, dtype, contiguous

    def get_device(self):
        return self.device_index

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 4096

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def element_size(self):
        return 1 if self.dtype == torch.uint8 else 4

    def dim(self):
        return len(self.shape)


B, S, STRIDE, P = 3, 2, 5, 40


def arguments(name):
    if name == "update":
        return dict(context_len=Fake(B), block_table=Fake(B, STRIDE), page_refs=Fake(P), need_len=Fake(B), capacity=Fake(B),
                    new_block_table=Fake(B, STRIDE), new_page_refs=Fake(P))
    if name == "fork":
        return dict(source=Fake(B), context_len=Fake(S), block_table=Fake(S, STRIDE), page_refs=Fake(P),
                    new_block_table=Fake(B, STRIDE), new_context_len=Fake(B), copy_src=Fake(B), copy_dst=Fake(B),
                    new_page_refs=Fake(P))
    if name == "compact":
        return dict(block_table=Fake(B, STRIDE), page_refs=Fake(P), new_place=Fake(P), move_src=Fake(P), move_dst=Fake(P),
                    counts=Fake(2), new_block_table=Fake(B, STRIDE), new_page_refs=Fake(P))
    pool = dict(dtype=torch.bfloat16)
    return dict(src=Fake(B), dst=Fake(B), count=Fake(1), k_pages=Fake(P, 2, 16, 64, **pool), v_pages=Fake(P, 2, 16, 64, **pool))


def call(name, args):
    more = dict(update=dict(page_size=16), fork=dict(page_size=16), compact={}, copy={})[name]
    if name != "copy":
        args.setdefault("workspace", Fake(4096, dtype=torch.uint8))
    getattr(ada, "adaserve_%s_pages" % name)(**args, **more)


CASES = [(name, at) for name in ("update", "fork", "compact", "copy") for at in arguments(name)]


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(ada, "_device_call", lambda name, device, stream, *args: made.append((name, device)))
    return made


@pytest.mark.parametrize("name", ["update", "fork", "compact", "copy"])
def test_device_tensors_are_taken(calls, name):
    call(name, arguments(name))
    assert calls == [("adaserve_%s_pages" % name, 0)]


@pytest.mark.parametrize("name,at", CASES)
@pytest.mark.parametrize("device", [-1, 1])
def test_one_tensor_elsewhere(calls, name, at, device):
    args = arguments(name)
    args[at].device_index = device
    with pytest.raises(ValueError, match="device"):
        call(name, args)
    assert not calls


@pytest.mark.parametrize("name", ["update", "fork", "compact", "copy"])
def test_all_tensors_on_the_host(calls, name):
    args = arguments(name)
    if name != "copy":
        args["workspace"] = Fake(4096, dtype=torch.uint8)
    for t in args.values():
        t.device_index = -1
    with pytest.raises(ValueError, match="device"):
        call(name, args)
    assert not calls


@pytest.mark.parametrize("name,at", CASES)
def test_strides(calls, name, at):
    args = arguments(name)
    args[at].contiguous = False
    with pytest.raises(ValueError, match="contiguous"):
        call(name, args)
    assert not calls


@pytest.mark.parametrize("name,at", [c for c in CASES if c[1] not in ("k_pages", "v_pages")])
def test_types(calls, name, at):
    args = arguments(name)
    args[at].dtype = torch.int64
    with pytest.raises(ValueError, match="int32"):
        call(name, args)
    assert not calls


ATTENTIONS = ["prompt", "decode", "tree"]


def attend(kind):
    """A call on tensors that are all on the host."""
    i32, rows = torch.int32, torch.zeros(B, 4, 64)
    lens, indptr = np.full(B, 20, np.int32), np.arange(B + 1, dtype=np.int32)
    args = dict(q=rows, k_pages=torch.zeros(P, 2, 16, 64), v_pages=torch.zeros(P, 2, 16, 64),
                block_table=torch.zeros(B, STRIDE, dtype=i32), out=torch.zeros(B, 4, 64), window=8, sinks=2, sm_scale=0.1)
    ip = torch.tensor(indptr)
    if kind == "prompt":
        args.update(token_indptr=ip, token_indptr_host=indptr, context_len=torch.tensor(lens), context_len_host=lens)
    elif kind == "decode":
        args.update(context_len=torch.tensor(lens), max_context=20)
    else:
        args.update(node_indptr=ip, node_indptr_host=indptr, parent=torch.full((B,), -1, dtype=i32), prefix_len=torch.tensor(lens),
                    prefix_len_host=lens, k_tree=torch.zeros(B, 2, 64), v_tree=torch.zeros(B, 2, 64))
    getattr(ada, "adaserve_window_%s_attn" % kind)(**args)


@pytest.mark.parametrize("kind", ATTENTIONS)
def test_attention_of_host_tensors(calls, kind):
    with pytest.raises(ValueError, match="device"):
        attend(kind)
    assert not calls


def test_pointers_of_a_host_tensor_before_device_ones():
    with pytest.raises(ValueError, match="device"):
        ada._pointers((Fake(3, device=-1), Fake(3)))
    with pytest.raises(ValueError, match="device"):
        ada._pointers((None, Fake(3)), (Fake(3, device=-1),))
    assert ada._pointers((None, Fake(3)), (Fake(3),)) == (0, [None, 4096])
