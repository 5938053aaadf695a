"""The attentions over a window and the cache's pages together, as a server runs
them: pages taken for prompts, the prompts appended and attended, beams forked from
them, tokens appended and attended one by one while pages leave the window, draft
trees verified and their paths committed, the pool compacted -- and every
attention equal to one over a cache that keeps everything, in fp64."""
import numpy as np
import pytest

import window_calls as calls
from oracle import window as oracle
from paged_calls import starts
from serving_inputs import PS, back, to_dev, typed
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def i32(x):
    return np.asarray(x, np.int32)


class Server:
    """Two layers' pools under one table; `told` holds every request's keys and values since its beginning."""

    def __init__(self, ada, dtype, rows, pages, window, sinks, stride=60, layers=2, hq=8, hkv=2, d=128):  # noqa: F811
        import torch
        self.ada, self.dtype, self.window, self.sinks, self.layers = ada, dtype, window, sinks, layers
        self.hq, self.hkv, self.d, self.scale, self.rows, self.stride, self.pages = hq, hkv, d, d ** -0.5, rows, stride, pages
        self.rng, self.held = np.random.default_rng(rows), True
        t = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.k, self.v = (torch.full((layers, pages, hkv, PS, d), float("nan"), dtype=t, device="cuda") for _ in range(2))
        self.table = torch.full((rows, stride), -1, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.refs[:7] = 1   # another program's, until the pool is compacted
        self.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.ws = torch.full((ada.adaserve_pages_workspace_bytes(rows, pages),), 255, dtype=torch.uint8, device="cuda")
        self.told = [[np.zeros((2, 0, hkv, d)) for _ in range(rows)] for _ in range(layers)]
        self.inv = to_dev((10000.0 ** (-np.arange(0, d, 2) / d)).astype(np.float32))

    def len_host(self):
        return back(self.lens)

    def take(self, more):
        import torch
        need = to_dev(i32(self.len_host() + more))
        cap = torch.full((self.rows,), -5, dtype=torch.int32, device="cuda")
        self.ada.adaserve_update_pages(context_len=self.lens, need_len=need, window=self.window, sinks=self.sinks, page_size=PS,
                                       block_table=self.table, page_refs=self.refs, capacity=cap, workspace=self.ws)
        torch.cuda.synchronize()
        assert (back(cap) == back(need)).all(), (back(cap), back(need))

    def rows_of(self, T):
        return typed(self.rng.standard_normal((T, self.hq + 2 * self.hkv, self.d)), self.dtype)

    def append(self, new):
        """New tokens of every request in all layers; their queries, layer by layer."""
        import torch
        indptr, T, before = to_dev(starts(new)), int(sum(new)), self.len_host()
        queries = []
        for i in range(self.layers):
            x = self.rows_of(T)
            dev = to_dev(x)
            q = torch.empty((T, self.hq, self.d), dtype=dev.dtype, device="cuda")
            k = torch.empty((T, self.hkv, self.d), dtype=dev.dtype, device="cuda")
            grown = torch.empty_like(self.lens)
            self.ada.adaserve_rope_append_kv(token_indptr=indptr, prefix_len=self.lens, q=dev[:, :self.hq],
                                             k=dev[:, self.hq:self.hq + self.hkv], v=dev[:, self.hq + self.hkv:], inv_freq=self.inv,
                                             q_out=q, k_out=k, k_pages=self.k[i], v_pages=self.v[i], block_table=self.table,
                                             new_prefix_len=grown)
            torch.cuda.synchronize()
            kv = np.stack([calls.widen(back(k)), calls.widen(x[:, self.hq + self.hkv:])])
            for r, a in enumerate(starts(new)[:-1]):
                self.told[i][r] = np.concatenate([self.told[i][r], kv[:, a:a + new[r]]], 1)
            queries.append(q)
        self.lens = grown
        assert (back(grown) == before + i32(new)).all()
        return queries

    def expect(self, i, q, new, extra=None):
        """fp64 over everything told: (output, size, reach).  extra: (trees, keys, values) of draft trees."""
        ctx = [x.shape[1] for x in self.told[i]]
        wide = -(-max(ctx) // PS)
        kp, vp = (np.zeros((self.rows * wide, self.hkv, PS, self.d)) for _ in range(2))
        table = np.arange(self.rows * wide).reshape(self.rows, wide)
        for r, kv in enumerate(self.told[i]):
            for t in range(ctx[r]):
                kp[table[r, t // PS], :, t % PS], vp[table[r, t // PS], :, t % PS] = kv[0, t], kv[1, t]
        q = back(q)
        if extra:
            trees, k, v = extra
            return oracle.tree_attention(q, trees.indptr, trees.parent, k, v, kp, vp, table, ctx, self.scale, self.window, self.sinks)
        return oracle.paged_attention(q, starts(new), kp, vp, table, ctx, self.scale, self.window, self.sinks)

    def attend_prompt(self, queries, new):
        import torch
        ctx, indptr = self.len_host(), starts(new)
        for i, q in enumerate(queries):
            need = self.ada.adaserve_window_prompt_attn_workspace_bytes(indptr, ctx, self.hq, self.hkv, self.d, PS, self.window,
                                                                        self.sinks, calls.code(self.ada, self.dtype))
            out = torch.empty_like(q)
            self.ada.adaserve_window_prompt_attn(
                token_indptr=to_dev(indptr), token_indptr_host=indptr, q=q, k_pages=self.k[i], v_pages=self.v[i],
                block_table=self.table, context_len=self.lens, context_len_host=ctx, window=self.window, sinks=self.sinks,
                sm_scale=self.scale, out=out, workspace=calls.workspace(need))
            torch.cuda.synchronize()
            calls.check("prompt", self.dtype, calls.widen(back(out)), self.expect(i, q, new), int(ctx.max()))

    def attend_token(self, queries):
        import torch
        ctx = self.len_host()
        most = self.stride * PS
        for i, q in enumerate(queries):
            need = self.ada.adaserve_window_decode_attn_workspace_bytes(self.rows, most, self.hq, self.hkv, self.d, PS, self.window,
                                                                        self.sinks, calls.code(self.ada, self.dtype))
            out = torch.empty_like(q)
            self.ada.adaserve_window_decode_attn(q=q, k_pages=self.k[i], v_pages=self.v[i], block_table=self.table,
                                                 context_len=self.lens, max_context=most, window=self.window, sinks=self.sinks,
                                                 sm_scale=self.scale, out=out, workspace=calls.workspace(need))
            torch.cuda.synchronize()
            calls.check("decode", self.dtype, calls.widen(back(out)), self.expect(i, q, [1] * self.rows), int(ctx.max()))

    def fork(self, source):
        import torch
        table, lens, src, dst = torch.empty_like(self.table), torch.empty_like(self.lens), *(torch.empty_like(self.lens) for _ in range(2))
        self.ada.adaserve_fork_pages(source=to_dev(i32(source)), context_len=self.lens, block_table=self.table, page_refs=self.refs,
                                     page_size=PS, new_block_table=table, new_context_len=lens, copy_src=src, copy_dst=dst,
                                     workspace=self.ws)
        self.ada.adaserve_copy_pages(src=src, dst=dst, k_pages=self.k, v_pages=self.v)
        torch.cuda.synchronize()
        assert (back(lens) == [self.len_host()[s] if s >= 0 else 0 for s in source]).all()
        self.table, self.lens = table, lens
        self.told = [[layer[s].copy() if s >= 0 else layer[0][:, :0] for s in source] for layer in self.told]

    def compact(self):
        import torch
        place, src, dst = (torch.empty_like(self.refs) for _ in range(3))
        counts = torch.empty(2, dtype=torch.int32, device="cuda")
        held, self.held = self.held, False
        if held:
            self.refs[:7] -= 1
        self.ada.adaserve_compact_pages(block_table=self.table, page_refs=self.refs, new_place=place, move_src=src, move_dst=dst,
                                        counts=counts, workspace=self.ws)
        self.ada.adaserve_copy_pages(src=src, dst=dst, count=counts[1:], k_pages=self.k, v_pages=self.v)
        torch.cuda.synchronize()
        used = int(counts[0])
        # nothing from there on is needed
        self.k[:, used:], self.v[:, used:] = float("nan"), float("nan")
        assert (int(counts[1]) > 0 or not held) and (back(self.refs)[:used] > 0).all() and (back(self.refs)[used:] == 0).all()

    def verify(self, nodes):
        """Draft trees over the cache; a root path of each becomes part of it."""
        import torch
        new = [nodes] * self.rows
        ctx = self.len_host()
        T = sum(new)
        accepted = to_dev(i32([3] * self.rows))
        grown = torch.empty_like(self.lens)
        for i in range(self.layers):
            trees = calls.Trees(self.rng, new, self.hkv, self.d, self.dtype)
            trees.parent = i32([[-1, 0, 1, 1, 0][n] if n < 5 else int(self.rng.integers(0, n)) for _ in new for n in range(nodes)])
            q = to_dev(typed(self.rng.standard_normal((T, self.hq, self.d)), self.dtype))
            out = torch.empty_like(q)
            need = self.ada.adaserve_window_tree_attn_workspace_bytes(trees.indptr, ctx, self.hq, self.hkv, self.d, PS, self.window,
                                                                      self.sinks, calls.code(self.ada, self.dtype))
            k, v = to_dev(trees.k), to_dev(trees.v)
            self.ada.adaserve_window_tree_attn(
                node_indptr=to_dev(trees.indptr), node_indptr_host=trees.indptr, parent=to_dev(trees.parent), q=q, k_tree=k,
                v_tree=v, k_pages=self.k[i], v_pages=self.v[i], block_table=self.table, prefix_len=self.lens, prefix_len_host=ctx,
                window=self.window, sinks=self.sinks, sm_scale=self.scale, out=out, workspace=calls.workspace(need))
            torch.cuda.synchronize()
            calls.check("tree", self.dtype, calls.widen(back(out)), self.expect(i, q, new, (trees, trees.k, trees.v)), int(ctx.max()) + nodes)
            self.ada.adaserve_commit_accepted_kv(
                node_indptr=to_dev(trees.indptr), accept_len=accepted, accept_nodes=to_dev(i32([[0, 1, 3]] * self.rows)), k_tree=k,
                v_tree=v, k_pages=self.k[i], v_pages=self.v[i], block_table=self.table, prefix_len=self.lens, new_prefix_len=grown)
            torch.cuda.synchronize()
            for r in range(self.rows):
                at = trees.indptr[r] + np.array([0, 1, 3])
                kv = np.stack([calls.widen(trees.k[at]), calls.widen(trees.v[at])])
                self.told[i][r] = np.concatenate([self.told[i][r], kv], 1)
        self.lens = grown
        assert (back(grown) == ctx + 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks,pages", [(70, 4, 170), (33, 0, 150), (200, 20, 5000)])
def test_a_server_over_a_window(ada, dtype, window, sinks, pages):  # noqa: F811
    s = Server(ada, dtype, 6, pages, window, sinks)
    new = [130, 1, 77, 300, 64, 16]
    s.take(new)
    s.attend_prompt(s.append(new), new)
    s.fork([3, 3, 0, 2, 3, 5])
    for step in range(3):
        s.take(1)
        s.attend_token(s.append([1] * 6))
        s.fork([[0, 0, 1, 3, 4, 5], [5, 4, 3, 2, 1, 0], [2, 2, -1, 0, 0, 1]][step])
    s.compact()
    s.take(3)
    s.verify(9)
    new = [20, 0, 3, 50, 1, 33]
    s.take(new)
    s.attend_prompt(s.append(new), new)
    s.compact()
    s.take(1)
    s.attend_token(s.append([1] * 6))
    # nothing but the rows' entries holds a page, and no row more than its window asks for
    table, refs = back(s.table), back(s.refs)
    assert (np.bincount(table[table >= 0], minlength=pages) == refs).all()
    assert ((table >= 0).sum(1) <= -(-sinks // PS) + (window + 2 * PS) // PS + 1).all()
    s.lens.fill_(-1)
    s.ada.adaserve_update_pages(context_len=s.lens, page_size=PS, block_table=s.table, page_refs=s.refs, workspace=s.ws)
    assert (back(s.refs) == 0).all() and (back(s.table) == -1).all()
