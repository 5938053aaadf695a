"""Refusals of the serving operators' entry points, on the host before any HIP
call (nothing here touches a device)."""
import ctypes
import os

import numpy as np
import pytest

import paper_2501_12162_amd as ada

FAKE = 0x1000   # never dereferenced: every call below fails validation first
SIZE_MAX = ctypes.c_size_t(-1).value
BAD, UNSUP, WS = ada.ADASERVE_ERR_INVALID_ARGUMENT, ada.ADASERVE_ERR_UNSUPPORTED, ada.ADASERVE_ERR_WORKSPACE
INT_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ada.library_path()):
        from paper_2501_12162_amd.build import build
        build()
    return ada.load_library()


def _append(lib, **kw):
    a = dict(B=2, T=5, indptr=FAKE, plen=FAKE, pos=None, q=0x10000, qs=512, k=0x20000, ks=256, v=0x30000, vs=256,
             inv=FAKE, rot=64, inter=0, hq=4, hkv=2, d=128, ps=16, dtype=ada.ADASERVE_BF16, qo=0x40000, ko=None,
             kp=0x50000, vp=0x60000, pages=4, bt=FAKE, bts=2, new=0x2000)
    a.update(kw)
    return lib.adaserve_rope_append_kv(
        a["B"], a["T"], a["indptr"], a["plen"], a["pos"], a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["inv"],
        a["rot"], a["inter"], a["hq"], a["hkv"], a["d"], a["ps"], a["dtype"], a["qo"], a["ko"], a["kp"], a["vp"],
        a["pages"], a["bt"], a["bts"], a["new"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), BAD), (dict(T=-1), BAD), (dict(dtype=5), BAD), (dict(d=0), BAD), (dict(d=100), UNSUP),
    (dict(d=1024), UNSUP), (dict(rot=-2), BAD), (dict(rot=130), BAD), (dict(rot=24), UNSUP), (dict(inter=2), BAD),
    (dict(hkv=0), BAD), (dict(hq=0), BAD), (dict(hkv=5000), UNSUP), (dict(ps=0), BAD), (dict(pages=-1), BAD),
    (dict(bts=-1), BAD), (dict(qo=None), BAD), (dict(q=None), BAD), (dict(kp=None), BAD), (dict(vp=None), BAD),
    (dict(kp=None, vp=None, ko=0x70000), BAD),                      # new_prefix_len without pages
    (dict(kp=None, vp=None, new=None), BAD),                        # k goes nowhere
    (dict(new=None), BAD), (dict(bt=None), BAD), (dict(indptr=None), BAD), (dict(plen=None), BAD),
    (dict(inv=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(q=None, qo=None, k=None), BAD),
    (dict(qs=511), BAD), (dict(qs=516), BAD), (dict(ks=8), BAD), (dict(vs=128), BAD), (dict(ks=2 ** 41), UNSUP),
    (dict(q=0x10008), BAD), (dict(k=0x20002), BAD), (dict(v=0x30004), BAD), (dict(qo=0x40008), BAD),
    (dict(ko=0x70004), BAD), (dict(kp=0x50008), BAD), (dict(vp=0x60002), BAD),
    (dict(qo=0x10010), BAD),                                        # shifted over its own input
    (dict(qs=1024, qo=0x10000), BAD),                               # in place needs dense rows
    (dict(qo=0x20000), BAD), (dict(ko=0x10000), BAD), (dict(ko=0x30000), BAD), (dict(ko=0x40000), BAD),
    (dict(new=FAKE + 4), BAD),                                      # overlaps prefix_len without being it
])
def test_append_refuses(lib, kw, code):
    assert _append(lib, **kw) == code and lib.adaserve_last_error()


def test_empty_calls_are_no_ops(lib):
    assert _append(lib, B=0) == 0
    assert _prompt(lib, ip=[0], ctx=[]) == 0
    assert _prompt(lib, ip=[0, 0, 0], ctx=[20, 0], q=None, out=None) == 0
    assert _decode(lib, B=0) == 0
    assert _sample(lib, rows=0, logits=None) == 0


def _prompt(lib, **kw):
    ip, ctx = np.asarray(kw.pop("ip", [0, 3, 5]), np.int32), np.asarray(kw.pop("ctx", [20, 5]), np.int32)
    a = dict(indptr=FAKE, q=FAKE, qs=1024, kp=FAKE, vp=FAKE, pages=4, bt=FAKE, bts=2, ctxd=FAKE, hq=8, hkv=2, d=128,
             ps=16, scale=0.1, dtype=ada.ADASERVE_BF16, out=FAKE, ws=None, wsb=0, iph=ip.ctypes.data, cth=ctx.ctypes.data)
    a.update(kw)
    return lib.adaserve_prompt_attn(
        int(ctx.size), a["indptr"], a["iph"], a["q"], a["qs"], a["kp"], a["vp"], a["pages"], a["bt"], a["bts"], a["ctxd"],
        a["cth"], a["hq"], a["hkv"], a["d"], a["ps"], a["scale"], a["dtype"], a["out"], a["ws"], a["wsb"], None)


COMMON = [
    (dict(hq=6, hkv=4), BAD), (dict(hq=0), BAD), (dict(hq=64, hkv=2), UNSUP), (dict(hq=8192, hkv=1024), UNSUP),
    (dict(d=80), UNSUP), (dict(ps=8), UNSUP), (dict(dtype=7), BAD), (dict(bts=-1), BAD), (dict(pages=-1), BAD),
    (dict(pages=0), BAD), (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(scale=0.0), UNSUP),
    (dict(scale=-0.1), UNSUP), (dict(q=None), BAD), (dict(out=None), BAD), (dict(ctxd=None), BAD), (dict(kp=None), BAD),
    (dict(vp=None), BAD), (dict(bt=None), BAD), (dict(q=FAKE + 8), BAD), (dict(out=FAKE + 2), BAD),
    (dict(kp=FAKE + 8), BAD), (dict(qs=1023), BAD), (dict(qs=1028), BAD), (dict(qs=2 ** 41), UNSUP),
]


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(ip=[1, 3, 5]), BAD), (dict(ip=[0, 5, 3]), BAD), (dict(ctx=[-1, 5]), BAD), (dict(ctx=[33, 5]), BAD),
    (dict(ctx=[2 ** 23, 5], bts=2 ** 20), UNSUP), (dict(indptr=None), BAD), (dict(iph=None), BAD), (dict(cth=None), BAD),
    (dict(ip=[0, 3, INT_MAX]), UNSUP),
])
def test_prompt_refuses(lib, kw, code):
    assert _prompt(lib, **kw) == code and lib.adaserve_last_error()


def _decode(lib, **kw):
    a = dict(B=2, q=FAKE, qs=1024, kp=FAKE, vp=FAKE, pages=4, bt=FAKE, bts=2, ctxd=FAKE, most=32, hq=8, hkv=2, d=128,
             ps=16, scale=0.1, dtype=ada.ADASERVE_BF16, out=FAKE, ws=None, wsb=0)
    a.update(kw)
    return lib.adaserve_decode_attn(
        a["B"], a["q"], a["qs"], a["kp"], a["vp"], a["pages"], a["bt"], a["bts"], a["ctxd"], a["most"], a["hq"], a["hkv"],
        a["d"], a["ps"], a["scale"], a["dtype"], a["out"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(B=-1), BAD), (dict(most=-1), BAD), (dict(most=33), BAD), (dict(most=2 ** 23, bts=2 ** 20), UNSUP),
    (dict(B=2 ** 28, hq=16, hkv=2, qs=2048), UNSUP),
])
def test_decode_refuses(lib, kw, code):
    assert _decode(lib, **kw) == code and lib.adaserve_last_error()


def _sample(lib, **kw):
    a = dict(logits=FAKE, stride=100, rows=3, vocab=100, dtype=ada.ADASERVE_F32, t=FAKE, k=FAKE, p=FAKE, m=FAKE, u=FAKE,
             out=FAKE, ws=FAKE * 16, wsb=1 << 40)
    a.update(kw)
    return lib.adaserve_sample(a["logits"], a["stride"], a["rows"], a["vocab"], a["dtype"], a["t"], a["k"], a["p"],
                               a["m"], a["u"], a["out"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), BAD), (dict(vocab=0), BAD), (dict(vocab=2 ** 20 + 1, stride=2 ** 21), UNSUP), (dict(dtype=2), BAD),
    (dict(stride=99), BAD), (dict(logits=None), BAD), (dict(u=None), BAD), (dict(out=None), BAD),
    (dict(logits=FAKE + 2), BAD), (dict(dtype=ada.ADASERVE_BF16, logits=FAKE + 1), BAD), (dict(t=FAKE + 1), BAD),
    (dict(k=FAKE + 2), BAD), (dict(p=FAKE + 2), BAD), (dict(m=FAKE + 2), BAD), (dict(u=FAKE + 2), BAD),
    (dict(out=FAKE + 2), BAD),
])
def test_sample_refuses(lib, kw, code):
    assert _sample(lib, **kw) == code and lib.adaserve_last_error()


def test_workspace_queries_refuse(lib):
    i32 = lambda a: np.asarray(a, np.int32)
    ip, ctx = i32([0, 3]), i32([20])
    prompt = lambda ip=ip, ctx=ctx, hq=8, hkv=2, d=128, ps=16, dt=1: lib.adaserve_prompt_attn_workspace_bytes(
        1, ip.ctypes.data, ctx.ctypes.data, hq, hkv, d, ps, dt)
    assert prompt() != SIZE_MAX
    for kw in (dict(hq=7), dict(d=96), dict(ps=32), dict(dt=3), dict(ip=i32([0, -1])), dict(ctx=i32([-1]))):
        assert prompt(**kw) == SIZE_MAX and lib.adaserve_last_error()
    decode = lambda B=4, most=100, hq=8, hkv=2, d=128, ps=16, dt=1: lib.adaserve_decode_attn_workspace_bytes(
        B, most, hq, hkv, d, ps, dt)
    assert decode() != SIZE_MAX
    for kw in (dict(B=-1), dict(most=-1), dict(most=2 ** 23), dict(hq=7), dict(d=96), dict(ps=32), dict(dt=3)):
        assert decode(**kw) == SIZE_MAX and lib.adaserve_last_error()
    assert lib.adaserve_sample_workspace_bytes(4, 1000, 0) != SIZE_MAX
    for args in ((-1, 1000, 0), (4, 0, 0), (4, 2 ** 20 + 1, 0), (4, 1000, 2)):
        assert lib.adaserve_sample_workspace_bytes(*args) == SIZE_MAX and lib.adaserve_last_error()
