"""Refusals of the attentions over a window and of the pages' entry points, on
the host before any HIP call (nothing here touches a device)."""
import ctypes
import os

import numpy as np
import pytest

import paper_2501_12162_amd as ada

FAKE = 0x10000   # never dereferenced: every call below fails validation first
SIZE_MAX = ctypes.c_size_t(-1).value
BAD, UNSUP, WS = ada.ADASERVE_ERR_INVALID_ARGUMENT, ada.ADASERVE_ERR_UNSUPPORTED, ada.ADASERVE_ERR_WORKSPACE
INT_MAX = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ada.library_path()):
        from paper_2501_12162_amd.build import build
        build()
    return ada.load_library()


def _prompt(lib, **kw):
    ip, ctx = np.asarray(kw.pop("ip", [0, 3, 5]), np.int32), np.asarray(kw.pop("ctx", [20, 5]), np.int32)
    a = dict(indptr=FAKE, q=FAKE, qs=1024, kp=FAKE, vp=FAKE, pages=4, bt=FAKE, bts=2, ctxd=FAKE, hq=8, hkv=2, d=128, ps=16,
             w=7, s=2, scale=0.1, dtype=ada.ADASERVE_BF16, out=FAKE, ws=None, wsb=0, iph=ip.ctypes.data, cth=ctx.ctypes.data)
    a.update(kw)
    return lib.adaserve_window_prompt_attn(
        int(ctx.size), a["indptr"], a["iph"], a["q"], a["qs"], a["kp"], a["vp"], a["pages"], a["bt"], a["bts"], a["ctxd"],
        a["cth"], a["hq"], a["hkv"], a["d"], a["ps"], a["w"], a["s"], a["scale"], a["dtype"], a["out"], a["ws"], a["wsb"], None)


def _decode(lib, **kw):
    a = dict(B=2, q=FAKE, qs=1024, kp=FAKE, vp=FAKE, pages=4, bt=FAKE, bts=2, ctxd=FAKE, most=32, hq=8, hkv=2, d=128, ps=16,
             w=7, s=2, scale=0.1, dtype=ada.ADASERVE_BF16, out=FAKE, ws=None, wsb=0)
    a.update(kw)
    return lib.adaserve_window_decode_attn(
        a["B"], a["q"], a["qs"], a["kp"], a["vp"], a["pages"], a["bt"], a["bts"], a["ctxd"], a["most"], a["hq"], a["hkv"],
        a["d"], a["ps"], a["w"], a["s"], a["scale"], a["dtype"], a["out"], a["ws"], a["wsb"], None)


def _tree(lib, **kw):
    ip, pl = np.asarray(kw.pop("ip", [0, 3, 5]), np.int32), np.asarray(kw.pop("pl", [20, 5]), np.int32)
    a = dict(indptr=FAKE, par=FAKE, q=FAKE, kt=FAKE, vt=FAKE, kp=FAKE, vp=FAKE, pages=4, bt=FAKE, bts=2, pld=FAKE, hq=8, hkv=2,
             d=128, ps=16, w=7, s=2, scale=0.1, dtype=ada.ADASERVE_BF16, out=FAKE, ws=None, wsb=0, iph=ip.ctypes.data,
             plh=pl.ctypes.data)
    a.update(kw)
    return lib.adaserve_window_tree_attn(
        int(pl.size), a["indptr"], a["iph"], a["par"], a["q"], a["kt"], a["vt"], a["kp"], a["vp"], a["pages"], a["bt"], a["bts"],
        a["pld"], a["plh"], a["hq"], a["hkv"], a["d"], a["ps"], a["w"], a["s"], a["scale"], a["dtype"], a["out"], a["ws"],
        a["wsb"], None)


COMMON = [
    (dict(w=0), BAD), (dict(w=-1), BAD), (dict(s=-1), BAD), (dict(w=-INT_MAX - 1), BAD),
    (dict(hq=6, hkv=4), BAD), (dict(hq=0), BAD), (dict(hq=64, hkv=2), UNSUP), (dict(d=80), UNSUP), (dict(ps=8), UNSUP),
    (dict(dtype=7), BAD), (dict(bts=-1), BAD), (dict(pages=-1), BAD), (dict(pages=0), BAD), (dict(scale=float("nan")), BAD),
    (dict(scale=float("inf")), BAD), (dict(scale=0.0), UNSUP), (dict(scale=-0.1), UNSUP), (dict(q=None), BAD),
    (dict(out=None), BAD), (dict(kp=None), BAD), (dict(vp=None), BAD), (dict(bt=None), BAD), (dict(q=FAKE + 8), BAD),
    (dict(out=FAKE + 2), BAD), (dict(kp=FAKE + 8), BAD),
]
ROWS = [(dict(ctxd=None), BAD), (dict(qs=1023), BAD), (dict(qs=1028), BAD), (dict(qs=2 ** 41), UNSUP)]


@pytest.mark.parametrize("kw,code", COMMON + ROWS + [
    (dict(ip=[1, 3, 5]), BAD), (dict(ip=[0, 5, 3]), BAD), (dict(ctx=[-1, 5]), BAD), (dict(ctx=[33, 5]), BAD),
    (dict(ctx=[2 ** 23, 5], bts=2 ** 20), UNSUP), (dict(indptr=None), BAD), (dict(iph=None), BAD), (dict(cth=None), BAD),
    (dict(ip=[0, 3, INT_MAX]), UNSUP),
])
def test_prompt_refuses(lib, kw, code):
    assert _prompt(lib, **kw) == code and lib.adaserve_last_error()


@pytest.mark.parametrize("kw,code", COMMON + ROWS + [
    (dict(B=-1), BAD), (dict(most=-1), BAD), (dict(most=33), BAD), (dict(most=2 ** 23, bts=2 ** 20), UNSUP),
    (dict(B=2 ** 28, hq=16, hkv=2, qs=2048), UNSUP),
])
def test_decode_refuses(lib, kw, code):
    assert _decode(lib, **kw) == code and lib.adaserve_last_error()


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(ip=[1, 3, 5]), BAD), (dict(ip=[0, 3, 3]), BAD), (dict(ip=[0, 3, 132]), UNSUP), (dict(pl=[-1, 5]), BAD),
    (dict(pl=[33, 5]), BAD), (dict(pl=[2 ** 23, 5], bts=2 ** 20), UNSUP), (dict(indptr=None), BAD), (dict(iph=None), BAD),
    (dict(plh=None), BAD), (dict(pld=None), BAD), (dict(par=None), BAD), (dict(kt=None), BAD), (dict(vt=None), BAD),
    (dict(kt=FAKE + 8), BAD), (dict(vt=FAKE + 4), BAD),
])
def test_tree_refuses(lib, kw, code):
    assert _tree(lib, **kw) == code and lib.adaserve_last_error()


def test_empty_calls_are_no_ops(lib):
    assert _prompt(lib, ip=[0], ctx=[]) == 0
    assert _prompt(lib, ip=[0, 0, 0], ctx=[20, 0], q=None, out=None) == 0
    assert _decode(lib, B=0) == 0
    assert _tree(lib, ip=[0], pl=[]) == 0


def test_workspace_queries(lib):
    ip, ctx = np.array([0, 3, 5], np.int32), np.array([20, 5], np.int32)
    p = (ip.ctypes.data, ctx.ctypes.data)
    for name in ("prompt", "tree"):
        query = getattr(lib, "adaserve_window_%s_attn_workspace_bytes" % name)
        assert query(2, *p, 8, 2, 128, 16, 5, 0, 1) != SIZE_MAX
        for bad in ((2, *p, 8, 2, 128, 16, 0, 0, 1), (2, *p, 8, 2, 128, 16, 5, -1, 1), (2, *p, 8, 3, 128, 16, 5, 0, 1),
                    (2, None, None, 8, 2, 128, 16, 5, 0, 1), (-1, *p, 8, 2, 128, 16, 5, 0, 1)):
            assert query(*bad) == SIZE_MAX and lib.adaserve_last_error()
    query = lib.adaserve_window_decode_attn_workspace_bytes
    assert query(4, 1000, 8, 2, 128, 16, 100, 4, 1) != SIZE_MAX
    for bad in ((4, 1000, 8, 2, 128, 16, 0, 4, 1), (4, 1000, 8, 2, 128, 16, 100, -4, 1), (4, -1, 8, 2, 128, 16, 100, 4, 1)):
        assert query(*bad) == SIZE_MAX
    query = lib.adaserve_pages_workspace_bytes
    assert query(0, 0) != SIZE_MAX and query(65536, 2 ** 23) != SIZE_MAX
    for bad in ((-1, 5), (5, -1), (65537, 5), (5, 2 ** 23 + 1)):
        assert query(*bad) == SIZE_MAX


def at(i):
    return FAKE + i * 0x100000


def _update(lib, **kw):
    a = dict(B=5, clen=at(1), need=at(2), w=9, s=1, ps=16, bt=at(3), bts=20, refs=at(4), pages=100, nbt=at(5), nrefs=at(6),
             cap=at(7), ws=at(8), wsb=1 << 20)
    a.update(kw)
    return lib.adaserve_update_pages(a["B"], a["clen"], a["need"], a["w"], a["s"], a["ps"], a["bt"], a["bts"], a["refs"], a["pages"],
                                     a["nbt"], a["nrefs"], a["cap"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), BAD), (dict(B=65537), UNSUP), (dict(pages=-1), BAD), (dict(pages=2 ** 23 + 1), UNSUP), (dict(bts=-1), BAD),
    (dict(bts=2 ** 24 + 1), UNSUP), (dict(ps=0), BAD), (dict(ps=65537), UNSUP), (dict(w=-1), BAD), (dict(s=-1), BAD),
    (dict(need=None), BAD), (dict(cap=None), BAD), (dict(clen=None), BAD), (dict(bt=None), BAD), (dict(refs=None), BAD),
    (dict(nbt=None), BAD), (dict(nrefs=None), BAD), (dict(ws=None), WS), (dict(wsb=100), WS), (dict(ws=at(8) + 4), BAD),
    (dict(clen=at(1) + 2), BAD), (dict(nrefs=at(4) + 4), BAD), (dict(nbt=at(3) + 8), BAD), (dict(nbt=at(4)), BAD),
    (dict(nrefs=at(5) + 16), BAD), (dict(cap=at(1)), BAD), (dict(cap=at(2)), BAD), (dict(nbt=at(1)), BAD), (dict(ws=at(6)), BAD),
])
def test_update_refuses(lib, kw, code):
    assert _update(lib, **kw) == code and lib.adaserve_last_error()


def _fork(lib, **kw):
    a = dict(S=4, B=5, src=at(1), clen=at(2), ps=16, bt=at(3), bts=20, refs=at(4), pages=100, nbt=at(5), nlen=at(6), nrefs=at(7),
             cs=at(8), cd=at(9), ws=at(10), wsb=1 << 20)
    a.update(kw)
    return lib.adaserve_fork_pages(a["S"], a["B"], a["src"], a["clen"], a["ps"], a["bt"], a["bts"], a["refs"], a["pages"], a["nbt"],
                                   a["nlen"], a["nrefs"], a["cs"], a["cd"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(S=-1), BAD), (dict(B=-1), BAD), (dict(S=65537), UNSUP), (dict(B=65537), UNSUP), (dict(pages=-1), BAD), (dict(bts=-1), BAD),
    (dict(ps=0), BAD), (dict(src=None), BAD), (dict(clen=None), BAD), (dict(bt=None), BAD), (dict(refs=None), BAD),
    (dict(nbt=None), BAD), (dict(nlen=None), BAD), (dict(nrefs=None), BAD), (dict(cs=None), BAD), (dict(cd=None), BAD),
    (dict(ws=None), WS), (dict(wsb=0), WS), (dict(nbt=at(3)), BAD), (dict(nlen=at(2)), BAD), (dict(nlen=at(2) + 8), BAD),
    (dict(cs=at(9)), BAD), (dict(cd=at(1)), BAD), (dict(nrefs=at(4) + 4), BAD), (dict(cs=at(8) + 1), BAD),
])
def test_fork_refuses(lib, kw, code):
    assert _fork(lib, **kw) == code and lib.adaserve_last_error()


def _compact(lib, **kw):
    a = dict(B=5, bt=at(1), bts=20, refs=at(2), pages=100, nbt=at(3), nrefs=at(4), place=at(5), ms=at(6), md=at(7), cnt=at(8),
             ws=at(9), wsb=1 << 20)
    a.update(kw)
    return lib.adaserve_compact_pages(a["B"], a["bt"], a["bts"], a["refs"], a["pages"], a["nbt"], a["nrefs"], a["place"], a["ms"],
                                      a["md"], a["cnt"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), BAD), (dict(pages=-1), BAD), (dict(bts=-1), BAD), (dict(B=65536, bts=2 ** 15), UNSUP), (dict(bt=None), BAD),
    (dict(refs=None), BAD), (dict(nbt=None), BAD), (dict(nrefs=None), BAD), (dict(place=None), BAD), (dict(ms=None), BAD),
    (dict(md=None), BAD), (dict(cnt=None), BAD), (dict(ws=None), WS), (dict(wsb=0), WS), (dict(nbt=at(1) + 4), BAD),
    (dict(nrefs=at(2) + 4), BAD), (dict(place=at(2)), BAD), (dict(ms=at(7)), BAD), (dict(cnt=at(4) + 8), BAD), (dict(md=at(1)), BAD),
])
def test_compact_refuses(lib, kw, code):
    assert _compact(lib, **kw) == code and lib.adaserve_last_error()


def _copy(lib, **kw):
    a = dict(n=3, src=at(1), dst=at(2), count=None, kp=at(3), vp=at(4), layers=2, stride=2 ** 20, pages=10, hkv=2, ps=16, d=64,
             dtype=ada.ADASERVE_BF16)
    a.update(kw)
    return lib.adaserve_copy_pages(a["n"], a["src"], a["dst"], a["count"], a["kp"], a["vp"], a["layers"], a["stride"], a["pages"],
                                   a["hkv"], a["ps"], a["d"], a["dtype"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), BAD), (dict(n=2 ** 23 + 1), UNSUP), (dict(layers=-1), BAD), (dict(layers=65537), UNSUP), (dict(pages=-1), BAD),
    (dict(pages=2 ** 23 + 1), UNSUP), (dict(hkv=0), BAD), (dict(hkv=4097), UNSUP), (dict(d=0), BAD), (dict(d=12), UNSUP),
    (dict(d=4104), UNSUP), (dict(ps=0), BAD), (dict(ps=65537), UNSUP), (dict(dtype=3), BAD), (dict(stride=2 * 16 * 64 * 10 - 8), BAD),
    (dict(stride=2 ** 20 + 4), BAD), (dict(stride=2 ** 48), UNSUP), (dict(pages=2 ** 23, hkv=4096, ps=65536, d=4096), UNSUP),
    (dict(src=None), BAD), (dict(dst=None), BAD), (dict(kp=None), BAD), (dict(vp=None), BAD), (dict(src=at(1) + 2), BAD),
    (dict(count=at(5) + 1), BAD), (dict(kp=at(3) + 8), BAD), (dict(vp=at(4) + 4), BAD),
])
def test_copy_refuses(lib, kw, code):
    assert _copy(lib, **kw) == code and lib.adaserve_last_error()


def test_copies_of_nothing(lib):
    assert _copy(lib, n=0, src=None, dst=None) == 0 and _copy(lib, layers=0) == 0 and _copy(lib, pages=0) == 0
