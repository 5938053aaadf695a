"""MI355X (gfx950) batched tree verification for SLO-customised speculative decoding.

Python binding of the C ABI in ``include/adaserve.h``.  The functions here
only marshal arguments (torch tensors -> device pointers, host mirrors ->
host pointers) and raise on a non-OK status; every step of the computation
runs in the library's HIP kernels.  The library must have been built
(``python -m paper_2501_12162_amd.build``); importing the binding does not
require it, but the first call fails loudly when it is missing.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

from .build import LIB_PATH

ADASERVE_OK = 0
ADASERVE_ERR_INVALID_ARGUMENT = 1
ADASERVE_ERR_UNSUPPORTED = 2
ADASERVE_ERR_WORKSPACE = 3
ADASERVE_ERR_DEVICE = 4
ADASERVE_F32 = 0
ADASERVE_BF16 = 1
MAX_TREE_NODES = 128
TREE_ATTN_SCRATCH_BYTES = 32 << 20

_STATUS_NAMES = {1: "INVALID_ARGUMENT", 2: "UNSUPPORTED", 3: "WORKSPACE", 4: "DEVICE"}

# Every function the header declares, with its ctypes signature.
_P, _I32, _I64, _F32, _SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
SIGNATURES = {
    "adaserve_tree_attn_workspace_bytes": (_SZ, [_I32, _P, _P, _I32, _I32, _I32, _I32, _I32]),
    "adaserve_tree_attn_verify": (_I32, [_I32, _P, _P, _P, _P, _P, _P, _P, _P, _I32, _P, _I32, _P, _P,
                                         _I32, _I32, _I32, _I32, _F32, _I32, _P, _P, _SZ, _P]),
    "adaserve_tree_attn_verify_noalloc": (_I32, [_I32, _P, _P, _P, _P, _P, _P, _P, _P, _I32, _P, _I32, _P,
                                                 _P, _I32, _I32, _I32, _I32, _F32, _I32, _P, _P]),
    "adaserve_tree_verify_step": (_I32, [_I32, _P, _P, _P, _P, _P, _P, _P, _P, _I32, _P, _I32, _P, _P,
                                         _I32, _I32, _I32, _I32, _F32, _I32, _P, _I64, _I32, _P, _I32,
                                         _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "adaserve_node_argmax": (_I32, [_P, _I64, _I32, _I32, _I32, _P, _P]),
    "adaserve_tree_accept": (_I32, [_I32, _I32, _P, _P, _P, _P, _I32, _P, _P, _P, _P]),
    "adaserve_commit_accepted_kv": (_I32, [_I32, _P, _P, _P, _I32, _P, _P, _P, _P, _I32, _P, _I32, _P,
                                           _I32, _I32, _I32, _I32, _P, _P]),
    "adaserve_select_trees": (_I32, [_I32, _I32, _P, _P, _P, _P, _I32, _I32, _I32, _P, _P, _P, _P]),
    "adaserve_beam_step_workspace_bytes": (_SZ, [_I32, _I32, _I32, _I32, _I32]),
    "adaserve_beam_step": (_I32, [_I32, _I32, _P, _I64, _I32, _I32, _P, _I32, _P, _P, _P, _P, _SZ, _P]),
    "adaserve_tree_accept_sampled_workspace_bytes": (_SZ, [_I32]),
    "adaserve_tree_accept_sampled": (_I32, [_I32, _I32, _P, _P, _P, _P, _P, _I64, _I32, _I32, _P, _P, _I32,
                                            _P, _P, _P, _P, _SZ, _P]),
    "adaserve_rope_append_kv": (_I32, [_I32, _I32, _P, _P, _P, _P, _I64, _P, _I64, _P, _I64, _P, _I32, _I32,
                                       _I32, _I32, _I32, _I32, _I32, _P, _P, _P, _P, _I32, _P, _I32, _P, _P]),
    "adaserve_prompt_attn_workspace_bytes": (_SZ, [_I32, _P, _P, _I32, _I32, _I32, _I32, _I32]),
    "adaserve_prompt_attn": (_I32, [_I32, _P, _P, _P, _I64, _P, _P, _I32, _P, _I32, _P, _P, _I32, _I32, _I32,
                                    _I32, _F32, _I32, _P, _P, _SZ, _P]),
    "adaserve_decode_attn_workspace_bytes": (_SZ, [_I32, _I32, _I32, _I32, _I32, _I32, _I32]),
    "adaserve_decode_attn": (_I32, [_I32, _P, _I64, _P, _P, _I32, _P, _I32, _P, _I32, _I32, _I32, _I32, _I32,
                                    _F32, _I32, _P, _P, _SZ, _P]),
    "adaserve_sample_workspace_bytes": (_SZ, [_I32, _I32, _I32]),
    "adaserve_sample": (_I32, [_P, _I64, _I32, _I32, _I32, _P, _P, _P, _P, _P, _P, _P, _SZ, _P]),
    "adaserve_last_error": (ctypes.c_char_p, []),
}

_lib = None


class AdaserveError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s (%d): %s" % (_STATUS_NAMES.get(status, "?"), status, message))
        self.status = status


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load ``libadaserve.so``; raises when it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or library_path()
    if not os.path.exists(p):
        raise ImportError("libadaserve.so is not built (%s); run `python -m paper_2501_12162_amd.build`" % p)
    lib = ctypes.CDLL(p)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if path is None:
        _lib = lib
    return lib


def library_path() -> str:
    """The in-tree build, or the build named by ADASERVE_LIBRARY (the CPU
    sanitizer run points it at an instrumented build of the same sources)."""
    return os.environ.get("ADASERVE_LIBRARY") or LIB_PATH


def _check(status: int) -> None:
    if status != ADASERVE_OK:
        msg = load_library().adaserve_last_error()
        raise AdaserveError(status, msg.decode() if msg else "")


def _dptr(t) -> Optional[int]:
    """Device pointer of a torch tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


def _host_i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a), dtype=np.int32)


def _stream(stream) -> Optional[int]:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return ADASERVE_BF16
    if t.dtype == torch.float32:
        return ADASERVE_F32
    raise ValueError("tensors must be bfloat16 or float32")


def adaserve_tree_attn_workspace_bytes(node_indptr_host, prefix_len_host, num_q_heads: int,
                                       num_kv_heads: int, head_dim: int, page_size: int,
                                       dtype: int) -> int:
    ip, pl = _host_i32(node_indptr_host), _host_i32(prefix_len_host)
    n = load_library().adaserve_tree_attn_workspace_bytes(
        int(pl.size), ip.ctypes.data, pl.ctypes.data, int(num_q_heads), int(num_kv_heads),
        int(head_dim), int(page_size), int(dtype))
    if n == ctypes.c_size_t(-1).value:
        _check(ADASERVE_ERR_INVALID_ARGUMENT)
    return int(n)


def adaserve_tree_attn_verify(*, node_indptr, node_indptr_host, parent, q, k_tree, v_tree,
                              k_pages, v_pages, block_table, prefix_len, prefix_len_host,
                              sm_scale: float, out, workspace=None, stream=None) -> None:
    """Tree attention; shapes: q/out [T, Hq, D], k_tree/v_tree [T, Hkv, D],
    k_pages/v_pages [P, Hkv, page_size, D], block_table [B, stride]."""
    ip, pl = _host_i32(node_indptr_host), _host_i32(prefix_len_host)
    T, Hq, D = q.shape
    Hkv = k_tree.shape[1]
    P, ps = k_pages.shape[0], k_pages.shape[2]
    bt_stride = block_table.shape[1] if block_table.dim() == 2 else 0
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = load_library().adaserve_tree_attn_verify(
        int(pl.size), _dptr(node_indptr), ip.ctypes.data, _dptr(parent), _dptr(q), _dptr(k_tree),
        _dptr(v_tree), _dptr(k_pages), _dptr(v_pages), int(P), _dptr(block_table), int(bt_stride),
        _dptr(prefix_len), pl.ctypes.data, int(Hq), int(Hkv), int(D), int(ps), float(sm_scale),
        _dtype_code(q), _dptr(out), _dptr(workspace), int(ws_bytes), _stream(stream))
    _check(st)


def adaserve_tree_attn_verify_noalloc(*, node_indptr, node_indptr_host, parent, q, k_tree, v_tree,
                                      k_pages, v_pages, block_table, prefix_len, prefix_len_host,
                                      sm_scale: float, out, stream=None) -> None:
    """Tree attention with the split-KV partials in the library's static
    scratch (no workspace argument, nothing allocated); arguments as
    ``adaserve_tree_attn_verify``."""
    ip, pl = _host_i32(node_indptr_host), _host_i32(prefix_len_host)
    T, Hq, D = q.shape
    Hkv = k_tree.shape[1]
    P, ps = k_pages.shape[0], k_pages.shape[2]
    bt_stride = block_table.shape[1] if block_table.dim() == 2 else 0
    st = load_library().adaserve_tree_attn_verify_noalloc(
        int(pl.size), _dptr(node_indptr), ip.ctypes.data, _dptr(parent), _dptr(q), _dptr(k_tree),
        _dptr(v_tree), _dptr(k_pages), _dptr(v_pages), int(P), _dptr(block_table), int(bt_stride),
        _dptr(prefix_len), pl.ctypes.data, int(Hq), int(Hkv), int(D), int(ps), float(sm_scale),
        _dtype_code(q), _dptr(out), _stream(stream))
    _check(st)


def adaserve_tree_verify_step(*, node_indptr, node_indptr_host, parent, q, k_tree, v_tree, k_pages, v_pages,
                              block_table, prefix_len, prefix_len_host, sm_scale: float, logits, vocab: int,
                              draft_tokens, max_accept: int, out, target_argmax, accept_len, accept_tokens,
                              accept_nodes, workspace=None, stream=None) -> None:
    """Attention, argmax and acceptance of one verification pass in one call;
    arguments as ``adaserve_tree_attn_verify``, ``adaserve_node_argmax`` and
    ``adaserve_tree_accept`` (logits [T, row_stride])."""
    ip, pl = _host_i32(node_indptr_host), _host_i32(prefix_len_host)
    T, Hq, D = q.shape
    Hkv = k_tree.shape[1]
    P, ps = k_pages.shape[0], k_pages.shape[2]
    bt_stride = block_table.shape[1] if block_table.dim() == 2 else 0
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = load_library().adaserve_tree_verify_step(
        int(pl.size), _dptr(node_indptr), ip.ctypes.data, _dptr(parent), _dptr(q), _dptr(k_tree),
        _dptr(v_tree), _dptr(k_pages), _dptr(v_pages), int(P), _dptr(block_table), int(bt_stride),
        _dptr(prefix_len), pl.ctypes.data, int(Hq), int(Hkv), int(D), int(ps), float(sm_scale),
        _dtype_code(q), _dptr(logits), int(logits.shape[1]), int(vocab), _dptr(draft_tokens), int(max_accept),
        _dptr(out), _dptr(target_argmax), _dptr(accept_len), _dptr(accept_tokens), _dptr(accept_nodes),
        _dptr(workspace), int(ws_bytes), _stream(stream))
    _check(st)


def adaserve_node_argmax(logits, vocab: int, argmax_out, stream=None) -> None:
    """Row argmax of ``logits`` [rows, row_stride] over columns ``0..vocab-1``."""
    rows, stride = logits.shape
    st = load_library().adaserve_node_argmax(_dptr(logits), int(stride), int(rows), int(vocab),
                                             _dtype_code(logits), _dptr(argmax_out), _stream(stream))
    _check(st)


def adaserve_tree_accept(*, node_indptr, parent, draft_tokens, target_argmax, max_accept: int,
                         accept_len, accept_tokens, accept_nodes, stream=None) -> None:
    """Longest accepted path per request (outputs [B], [B, max_accept], [B, max_accept])."""
    B = node_indptr.shape[0] - 1
    st = load_library().adaserve_tree_accept(
        int(B), int(parent.shape[0]), _dptr(node_indptr), _dptr(parent), _dptr(draft_tokens),
        _dptr(target_argmax), int(max_accept), _dptr(accept_len), _dptr(accept_tokens),
        _dptr(accept_nodes), _stream(stream))
    _check(st)


def adaserve_commit_accepted_kv(*, node_indptr, accept_len, accept_nodes, k_tree, v_tree, k_pages,
                                v_pages, block_table, prefix_len, new_prefix_len, stream=None) -> None:
    """Write the accepted paths' K/V rows into the paged cache at L_r .. L_r + len - 1.
    accept_nodes [B, max_accept]; k_tree/v_tree [T, Hkv, D]; k_pages/v_pages [P, Hkv, ps, D]."""
    B = node_indptr.shape[0] - 1
    _, Hkv, D = k_tree.shape
    P, ps = k_pages.shape[0], k_pages.shape[2]
    bt_stride = block_table.shape[1] if block_table.dim() == 2 else 0
    st = load_library().adaserve_commit_accepted_kv(
        int(B), _dptr(node_indptr), _dptr(accept_len), _dptr(accept_nodes), int(accept_nodes.shape[1]),
        _dptr(k_tree), _dptr(v_tree), _dptr(k_pages), _dptr(v_pages), int(P), _dptr(block_table),
        int(bt_stride), _dptr(prefix_len), int(Hkv), int(D), int(ps), _dtype_code(k_tree),
        _dptr(new_prefix_len), _stream(stream))
    _check(st)


def adaserve_select_trees(*, cand_indptr, cand_parent, cand_prob, need, budget: int, n_max: int,
                          tree_size, tree_parent, tree_cand, stream=None) -> None:
    """Draft trees from candidate trees (tree_parent / tree_cand [B, max_nodes], max_nodes >= 128)."""
    B = cand_indptr.shape[0] - 1
    st = load_library().adaserve_select_trees(
        int(B), int(cand_prob.shape[0]), _dptr(cand_indptr), _dptr(cand_parent), _dptr(cand_prob),
        _dptr(need), int(budget), int(n_max), int(tree_parent.shape[1]), _dptr(tree_size),
        _dptr(tree_parent), _dptr(tree_cand), _stream(stream))
    _check(st)



def adaserve_beam_step_workspace_bytes(num_requests: int, beam_in: int, vocab: int, beam_out: int,
                                       dtype: int) -> int:
    n = load_library().adaserve_beam_step_workspace_bytes(int(num_requests), int(beam_in), int(vocab),
                                                          int(beam_out), int(dtype))
    if n == ctypes.c_size_t(-1).value:
        _check(ADASERVE_ERR_INVALID_ARGUMENT)
    return int(n)


def adaserve_beam_step(*, logits, vocab: int, beam_logprob, out_parent, out_token, out_logprob,
                       workspace, stream=None) -> None:
    """One beam-search step.  logits [num_requests * beam_in, row_stride];
    beam_logprob [num_requests, beam_in] float32; outputs [num_requests, beam_out]."""
    B, w_in = beam_logprob.shape
    rows, stride = logits.shape
    if rows != B * w_in:
        raise ValueError("logits has %d rows, beam_logprob asks for %d" % (rows, B * w_in))
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = load_library().adaserve_beam_step(
        int(B), int(w_in), _dptr(logits), int(stride), int(vocab), _dtype_code(logits), _dptr(beam_logprob),
        int(out_parent.shape[1]), _dptr(out_parent), _dptr(out_token), _dptr(out_logprob), _dptr(workspace),
        int(ws_bytes), _stream(stream))
    _check(st)


def adaserve_tree_accept_sampled_workspace_bytes(total_nodes: int) -> int:
    n = load_library().adaserve_tree_accept_sampled_workspace_bytes(int(total_nodes))
    if n == ctypes.c_size_t(-1).value:
        _check(ADASERVE_ERR_INVALID_ARGUMENT)
    return int(n)


def adaserve_tree_accept_sampled(*, node_indptr, parent, draft_tokens, target_logits, draft_logits, vocab: int,
                                 u_accept, u_bonus, max_accept: int, accept_len, accept_tokens, accept_nodes,
                                 workspace, stream=None) -> None:
    """Sampled-decoding tree verification; logits [T, row_stride] (temperature applied),
    u_accept / u_bonus [T] float32; workspace of adaserve_tree_accept_sampled_workspace_bytes(T)
    bytes; outputs as adaserve_tree_accept."""
    B = node_indptr.shape[0] - 1
    T, stride = target_logits.shape
    if draft_logits.shape != target_logits.shape or draft_logits.dtype != target_logits.dtype:
        raise ValueError("draft_logits must match target_logits in shape and dtype")
    st = load_library().adaserve_tree_accept_sampled(
        int(B), int(parent.shape[0]), _dptr(node_indptr), _dptr(parent), _dptr(draft_tokens),
        _dptr(target_logits), _dptr(draft_logits), int(stride), int(vocab), _dtype_code(target_logits),
        _dptr(u_accept), _dptr(u_bonus), int(max_accept), _dptr(accept_len), _dptr(accept_tokens),
        _dptr(accept_nodes), _dptr(workspace), int(0 if workspace is None else workspace.numel() * workspace.element_size()),
        _stream(stream))
    _check(st)


def _pointers(dense, strided=()):
    """The tensors' device, and the pointers of the dense ones (None -> NULL)."""
    device, pointers = -1, []
    for t in dense:
        if t is None:
            pointers.append(None)
            continue
        at = t.get_device()
        if at != device:
            if at < 0 or device >= 0:
                raise ValueError("expected a device tensor" if at < 0 else "tensors are on different devices")
            device = at
        if not t.is_contiguous():
            raise ValueError("expected a contiguous tensor")
        pointers.append(t.data_ptr())
    for t in strided:
        if t is not None and t.get_device() != device:
            raise ValueError("expected a device tensor" if t.get_device() < 0 else "tensors are on different devices")
    return device, pointers


def _device_call(name: str, device: int, stream, *args) -> None:
    """Calls entry point ``name`` on a device: its current stream where none is given, and the device made
    current for the call where it is not."""
    import torch
    fn = getattr(load_library(), name)
    s = (torch.cuda.current_stream(device) if stream is None else stream).cuda_stream
    if device == torch.cuda.current_device():
        st = fn(*args, s)
    else:
        with torch.cuda.device(device):
            st = fn(*args, s)
    if st != ADASERVE_OK:
        _check(st)


def _rows(t, name: str):
    """(pointer, elements between rows) of a [rows, heads, dim] tensor whose rows are dense."""
    if t is None:
        return None, 0
    (rows, heads, dim), (step, head_step, one) = t.shape, t.stride()
    # (the step of an axis of one entry means nothing)
    if rows and ((dim > 1 and one != 1) or (heads > 1 and head_step != dim)):
        raise ValueError("%s must have dense heads" % name)
    return t.data_ptr(), step if rows > 1 else heads * dim


def _typed(t, dtype, name: str) -> None:
    if t is not None and t.dtype != dtype:
        raise ValueError("%s must be %s" % (name, dtype))


def _bytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def adaserve_rope_append_kv(*, token_indptr, prefix_len, q=None, k=None, v=None, inv_freq=None, interleaved=False,
                            positions=None, q_out=None, k_out=None, k_pages=None, v_pages=None, block_table=None,
                            new_prefix_len=None, stream=None) -> None:
    """Rotates q [T, Hq, D] and k [T, Hkv, D] and appends k, v to the pages [P, Hkv, page_size, D].
    Rows of q, k, v may lie apart (slices of a projection's output); inv_freq [rotary_dim / 2] float32."""
    import torch
    main = k if k is not None else q
    if main is None:
        raise ValueError("neither q nor k is given")
    B = token_indptr.shape[0] - 1
    T, heads, D = main.shape
    hq = 0 if q is None else q.shape[1]
    hkv = 1 if k is None else heads
    pages, ps = 0, 1
    if k_pages is not None:
        pages, page_heads, ps, page_dim = k_pages.shape
        if k is None or page_heads != hkv or page_dim != D or v_pages is None or v_pages.shape != k_pages.shape:
            raise ValueError("k_pages and v_pages must be [pages, %d, page_size, %d]" % (hkv, D))
    for t, name, like, h in ((q, "q", main, hq), (v, "v", k, hkv), (q_out, "q_out", q, hq), (k_out, "k_out", k, hkv)):
        if t is not None:
            if like is None or t.shape != (T, h, D):
                raise ValueError("%s does not fit the tokens, heads and head dim of the other rows" % name)
            _typed(t, main.dtype, name)
    for t, name in ((k_pages, "k_pages"), (v_pages, "v_pages")):
        _typed(t, main.dtype, name)
    for t, name, n in ((token_indptr, "token_indptr", None), (prefix_len, "prefix_len", B), (positions, "positions", T),
                       (block_table, "block_table", B), (new_prefix_len, "new_prefix_len", B)):
        _typed(t, torch.int32, name)
        if t is not None and n is not None and t.shape[0] != n:
            raise ValueError("%s has %d rows, expected %d" % (name, t.shape[0], n))
    _typed(inv_freq, torch.float32, "inv_freq")
    (qp, qs), (kp, ks), (vp, vs) = _rows(q, "q"), _rows(k, "k"), _rows(v, "v")
    device, (ip, pl, pos, inv, qo, ko, kpg, vpg, bt, new) = _pointers(
        (token_indptr, prefix_len, positions, inv_freq, q_out, k_out, k_pages, v_pages, block_table, new_prefix_len),
        (q, k, v))
    _device_call("adaserve_rope_append_kv", device, stream, B, T, ip, pl, pos, qp, qs, kp, ks, vp, vs, inv,
                 0 if inv_freq is None else 2 * inv_freq.shape[0], int(interleaved), hq, hkv, D, ps, _dtype_code(main),
                 qo, ko, kpg, vpg, pages, bt, 0 if block_table is None else block_table.shape[1], new)


def _check_paged(q, k_pages, v_pages, block_table, context_len, out, requests) -> None:
    import torch
    if v_pages.shape != k_pages.shape or k_pages.dim() != 4 or k_pages.shape[3] != q.shape[2]:
        raise ValueError("k_pages and v_pages must be [pages, kv-heads, page_size, %d]" % q.shape[2])
    if out.shape != q.shape:
        raise ValueError("out must have q's shape")
    for t, name in ((k_pages, "k_pages"), (v_pages, "v_pages"), (out, "out")):
        _typed(t, q.dtype, name)
    _typed(block_table, torch.int32, "block_table")
    _typed(context_len, torch.int32, "context_len")
    if block_table.dim() != 2 or block_table.shape[0] != requests or context_len.shape[0] != requests:
        raise ValueError("block_table and context_len must have %d rows" % requests)


def adaserve_prompt_attn_workspace_bytes(token_indptr_host, context_len_host, num_q_heads: int, num_kv_heads: int,
                                         head_dim: int, page_size: int, dtype: int) -> int:
    ip, cl = _host_i32(token_indptr_host), _host_i32(context_len_host)
    n = load_library().adaserve_prompt_attn_workspace_bytes(cl.size, ip.ctypes.data, cl.ctypes.data, num_q_heads,
                                                            num_kv_heads, head_dim, page_size, dtype)
    if n == ctypes.c_size_t(-1).value:
        _check(ADASERVE_ERR_INVALID_ARGUMENT)
    return n


def adaserve_prompt_attn(*, token_indptr, token_indptr_host, q, k_pages, v_pages, block_table, context_len,
                         context_len_host, sm_scale: float, out, workspace=None, stream=None) -> None:
    """Causal attention of packed prompts; q/out [T, Hq, D] (rows of q may lie apart), k_pages/v_pages
    [P, Hkv, page_size, D], block_table [B, stride], context_len [B] with the rows' own keys counted."""
    import torch
    ip, cl = _host_i32(token_indptr_host), _host_i32(context_len_host)
    B = cl.size
    T, Hq, D = q.shape
    if ip.size != B + 1 or token_indptr.shape[0] != B + 1 or (B and T < ip[B]):
        raise ValueError("token_indptr must have %d entries, the last at most %d" % (B + 1, T))
    _check_paged(q, k_pages, v_pages, block_table, context_len, out, B)
    _typed(token_indptr, torch.int32, "token_indptr")
    qp, qs = _rows(q, "q")
    device, (tip, kp, vp, bt, clen, o, ws) = _pointers(
        (token_indptr, k_pages, v_pages, block_table, context_len, out, workspace), (q,))
    _device_call("adaserve_prompt_attn", device, stream, B, tip, ip.ctypes.data, qp, qs, kp, vp, k_pages.shape[0], bt,
                 block_table.shape[1], clen, cl.ctypes.data, Hq, k_pages.shape[1], D, k_pages.shape[2], sm_scale,
                 _dtype_code(q), o, ws, _bytes(workspace))


def adaserve_decode_attn_workspace_bytes(num_requests: int, max_context: int, num_q_heads: int, num_kv_heads: int,
                                         head_dim: int, page_size: int, dtype: int) -> int:
    n = load_library().adaserve_decode_attn_workspace_bytes(num_requests, max_context, num_q_heads, num_kv_heads,
                                                            head_dim, page_size, dtype)
    if n == ctypes.c_size_t(-1).value:
        _check(ADASERVE_ERR_INVALID_ARGUMENT)
    return n


def adaserve_decode_attn(*, q, k_pages, v_pages, block_table, context_len, max_context: int, sm_scale: float, out,
                         workspace=None, stream=None) -> None:
    """Attention of one token per request; q/out [B, Hq, D], context_len [B] (device) at most max_context."""
    B, Hq, D = q.shape
    _check_paged(q, k_pages, v_pages, block_table, context_len, out, B)
    qp, qs = _rows(q, "q")
    device, (kp, vp, bt, clen, o, ws) = _pointers((k_pages, v_pages, block_table, context_len, out, workspace), (q,))
    _device_call("adaserve_decode_attn", device, stream, B, qp, qs, kp, vp, k_pages.shape[0], bt, block_table.shape[1],
                 clen, max_context, Hq, k_pages.shape[1], D, k_pages.shape[2], sm_scale, _dtype_code(q), o, ws,
                 _bytes(workspace))


def adaserve_sample_workspace_bytes(num_rows: int, vocab: int, dtype: int) -> int:
    n = load_library().adaserve_sample_workspace_bytes(num_rows, vocab, dtype)
    if n == ctypes.c_size_t(-1).value:
        _check(ADASERVE_ERR_INVALID_ARGUMENT)
    return n


def adaserve_sample(*, logits, vocab: int, u, out_token, temperature=None, top_k=None, top_p=None, min_p=None,
                    workspace=None, stream=None) -> None:
    """A token per row of logits [rows, >= vocab] (rows may lie apart); temperature, top_p, min_p, u [rows]
    float32, top_k and out_token [rows] int32."""
    import torch
    rows, width = logits.shape
    if vocab > width:
        raise ValueError("vocab %d > %d columns" % (vocab, width))
    if width > 1 and logits.stride(1) != 1:
        raise ValueError("logits must have dense rows")
    for t, dtype, name in ((temperature, torch.float32, "temperature"), (top_k, torch.int32, "top_k"),
                           (top_p, torch.float32, "top_p"), (min_p, torch.float32, "min_p"), (u, torch.float32, "u"),
                           (out_token, torch.int32, "out_token")):
        _typed(t, dtype, name)
        if t is not None and t.numel() != rows:
            raise ValueError("%s has %d entries, expected %d" % (name, t.numel(), rows))
    device, (t, k, p, m, up, out, ws) = _pointers((temperature, top_k, top_p, min_p, u, out_token, workspace), (logits,))
    _device_call("adaserve_sample", device, stream, logits.data_ptr(), logits.stride(0) if rows > 1 else width, rows,
                 vocab, _dtype_code(logits), t, k, p, m, up, out, ws, _bytes(workspace))
