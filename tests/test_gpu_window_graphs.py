"""Captured calls of the attentions over a window, prompts and trees too: graphs that share a workspace,
replayed in turn with eager calls between them, and calls on two streams at once."""
import numpy as np
import pytest

import window_calls as calls
from paged_calls import starts
from serving_inputs import PS, back, to_dev
from test_gpu_paged_attention import ada  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
DTYPES = ["bf16", "f32"]
D, HQ, HKV, SINKS, SCALE = 128, 8, 2, 4, 0.09
NEW, CTX = {"prompt": [9, 20], "decode": [1, 1], "tree": [9, 20]}, [900, 2100]


class Call:
    """A call of one kind on tensors of its own, and what it gives in fp64."""

    def __init__(self, ada, kind, dtype, seed, window):  # noqa: F811
        import torch
        self.kind, self.dtype, self.entry = kind, dtype, getattr(ada, "adaserve_window_%s_attn" % kind)
        rng = np.random.default_rng(seed)
        new, ctx = NEW[kind], np.asarray(CTX, np.int32)
        cache, trees, q = calls.case(rng, kind, dtype, D, HQ, HKV, new, CTX, window, SINKS)
        self.expected = calls.expected(kind, cache, trees, q, new, CTX, SCALE, window, SINKS)
        indptr, code = starts(new), calls.code(ada, dtype)
        rows = to_dev(q)
        self.out = torch.empty_like(rows)
        self.args = dict(q=rows, k_pages=to_dev(cache.k), v_pages=to_dev(cache.v), block_table=to_dev(cache.table), window=window,
                         sinks=SINKS, sm_scale=SCALE, out=self.out)
        query = getattr(ada, "adaserve_window_%s_attn_workspace_bytes" % kind)
        shape = (HQ, HKV, D, PS, window, SINKS, code)
        if kind == "decode":
            self.args.update(context_len=to_dev(ctx), max_context=max(CTX))
            self.need = query(len(CTX), max(CTX), *shape)
        elif kind == "prompt":
            self.args.update(token_indptr=to_dev(indptr), token_indptr_host=indptr, context_len=to_dev(ctx), context_len_host=ctx)
            self.need = query(indptr, ctx, *shape)
        else:
            self.args.update(node_indptr=to_dev(indptr), node_indptr_host=indptr, parent=to_dev(trees.parent), prefix_len=to_dev(ctx),
                             prefix_len_host=ctx, k_tree=to_dev(trees.k), v_tree=to_dev(trees.v))
            self.need = query(indptr, ctx, *shape)

    def __call__(self, workspace, stream=None):
        self.entry(workspace=workspace, stream=stream, **self.args)

    def take(self):
        got = calls.widen(back(self.out))
        self.out.fill_(7)
        return got

    def check(self, got):
        calls.check(self.kind, self.dtype, got, self.expected, max(CTX) + 40)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [300, 1500])
def test_graphs_that_share_a_workspace(ada, window, dtype):  # noqa: F811
    import torch
    each = [Call(ada, kind, dtype, 20 + i, window) for i, kind in enumerate(("prompt", "decode", "tree"))]
    if dtype == "bf16" and window == 1500:   # (few rows over many keys: all are split)
        assert all(c.need > 0 for c in each)
    shared = torch.full((max(max(c.need for c in each), 1),), 255, dtype=torch.uint8, device="cuda")
    eager = []
    for c in each:
        print("eager", c.kind, dtype, "workspace", c.need, flush=True)
        c(shared)
        torch.cuda.synchronize()
        eager.append(c.take())
        c.check(eager[-1])
    graphs = []
    for c in each:
        print("capture", c.kind, dtype, flush=True)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c(shared)
    for step in range(4):
        for i in (0, 1, 2, 1, 0, 2):
            print("replay", step, each[i].kind, flush=True)
            graphs[i].replay()
            each[(i + step) % 3](shared)   # (an eager one behind it, of the same or another kind)
        torch.cuda.synchronize()
        for i, c in enumerate(each):
            assert np.array_equal(c.take(), eager[i])
        shared.fill_(step)                 # nothing of it outlives a call
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["prompt", "decode", "tree"])
def test_two_streams_at_once(ada, kind, dtype):  # noqa: F811
    import torch
    pair = [Call(ada, kind, dtype, 30 + i, 1500) for i in range(2)]
    spaces = [calls.workspace(c.need) for c in pair]
    streams = [torch.cuda.Stream() for _ in pair]
    torch.cuda.synchronize()
    print("two streams", kind, dtype, flush=True)
    for _ in range(8):
        for c, ws, s in zip(pair, spaces, streams):
            c(ws, s)
    for s in streams:
        s.synchronize()
    for c in pair:
        c.check(c.take())
