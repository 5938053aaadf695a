"""The serving operators together, as a server runs them: prompts rotated and
appended, attended, their first token drawn, then tokens appended, attended and
drawn one by one, eagerly and from a captured graph, on streams of their own.
Each step is checked against the fp64 oracle on what stands in the device's
buffers at that point."""
import numpy as np
import pytest

from oracle import serving
from serving_inputs import PS, Cache, attention_bound, back, to_dev, typed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ada():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2501_12162_amd as ada
    ada.load_library()
    return ada


class Server:
    """One layer that serves: a token's embedding row is its projected queries,
    keys and values, and the attention's output is its logits."""

    def __init__(self, ada, seed, lens, dtype, hq=8, hkv=2, d=128, vocab=1000, steps=8):
        import torch
        self.ada, self.dtype, self.hq, self.hkv, self.d, self.vocab = ada, dtype, hq, hkv, d, vocab
        rng = np.random.default_rng(seed)
        self.B = B = len(lens)
        self.code = ada.ADASERVE_BF16 if dtype == "bf16" else ada.ADASERVE_F32
        cache = Cache(rng, np.zeros(B, int), hkv, d, dtype, reach=np.asarray(lens) + steps)
        self.table_host = cache.table
        self.kp, self.vp, self.table = to_dev(cache.k), to_dev(cache.v), to_dev(cache.table)
        self.embed = to_dev(typed(rng.standard_normal((vocab, hq + 2 * hkv, d)), dtype))
        self.inv = to_dev((10000.0 ** (-np.arange(0, d, 2) / d)).astype(np.float32))
        self.indptr_host = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.prompt = to_dev(rng.integers(0, vocab, int(self.indptr_host[-1])).astype(np.int32))
        self.indptr, self.one = to_dev(self.indptr_host), to_dev(np.arange(B + 1, dtype=np.int32))
        self.lens, self.lens_host = to_dev(np.zeros(B, np.int32)), np.asarray(lens, np.int32)
        self.most = int(max(lens)) + steps
        self.scale = d ** -0.5
        ws = lambda n: torch.full((max(n, 1),), 255, dtype=torch.uint8, device="cuda")
        self.ws_prompt = ws(ada.adaserve_prompt_attn_workspace_bytes(self.indptr_host, self.lens_host, hq, hkv, d, PS, self.code))
        self.ws_decode = ws(ada.adaserve_decode_attn_workspace_bytes(B, self.most, hq, hkv, d, PS, self.code))
        self.ws_sample = ws(ada.adaserve_sample_workspace_bytes(B, vocab, self.code))
        self.token = torch.full((B,), -7, dtype=torch.int32, device="cuda")
        self.u = torch.zeros(B, device="cuda")
        self.par = dict(temperature=np.full(B, 0.05, np.float32), top_k=np.array([0, 50, 7, 1] * B, np.int32)[:B],
                        top_p=np.array([0.9, 1.0, 0.5] * B, np.float32)[:B], min_p=np.array([0, 0.01] * B, np.float32)[:B])
        self.par_dev = {k: to_dev(v) for k, v in self.par.items()}

    def append(self, x, indptr):
        """Rotated queries; keys and values stored, the lengths grown in place."""
        import torch
        hq, hkv = self.hq, self.hkv
        q = torch.empty((x.shape[0], hq, self.d), dtype=x.dtype, device="cuda")
        self.ada.adaserve_rope_append_kv(token_indptr=indptr, prefix_len=self.lens, q=x[:, :hq], k=x[:, hq:hq + hkv],
                                         v=x[:, hq + hkv:], inv_freq=self.inv, q_out=q, k_pages=self.kp, v_pages=self.vp,
                                         block_table=self.table, new_prefix_len=self.lens)
        return q

    def draw(self, rows):
        self.ada.adaserve_sample(logits=rows.reshape(self.B, self.hq * self.d), vocab=self.vocab, u=self.u,
                                 out_token=self.token, workspace=self.ws_sample, **self.par_dev)

    def prefill(self):
        import torch
        self.q = self.append(torch.index_select(self.embed, 0, self.prompt), self.indptr)
        self.out = torch.empty_like(self.q)
        self.ada.adaserve_prompt_attn(token_indptr=self.indptr, token_indptr_host=self.indptr_host, q=self.q,
                                      k_pages=self.kp, v_pages=self.vp, block_table=self.table, context_len=self.lens,
                                      context_len_host=self.lens_host, sm_scale=self.scale, out=self.out,
                                      workspace=self.ws_prompt)
        self.rows = torch.index_select(self.out, 0, self.indptr[1:] - 1)
        self.draw(self.rows)

    def step(self):
        import torch
        self.q = self.append(torch.index_select(self.embed, 0, self.token), self.one)
        self.out = torch.empty_like(self.q)
        self.ada.adaserve_decode_attn(q=self.q, k_pages=self.kp, v_pages=self.vp, block_table=self.table,
                                      context_len=self.lens, max_context=self.most, sm_scale=self.scale, out=self.out,
                                      workspace=self.ws_decode)
        self.rows = self.out
        self.draw(self.rows)

    def check(self, indptr_host, lens):
        """The buffers of the step that ran last against the oracle on its inputs."""
        assert back(self.lens).tolist() == list(lens)
        q, kp, vp = back(self.q), back(self.kp), back(self.vp)
        ref, size, reach = serving.paged_attention(q, indptr_host, kp, vp, self.table_host, lens, self.scale)
        got = serving.widen(back(self.out))
        assert (np.abs(got - ref) <= attention_bound(self.dtype, ref, size, reach, int(max(lens)), self.d)).all()
        logits = back(self.rows).reshape(self.B, -1)
        assert back(self.token).tolist() == serving.sample(logits, self.vocab, u=back(self.u), **self.par).tolist()

    def stored(self, tokens):
        """Keys and values in the pages: what the oracle makes of the tokens so far (lists per request)."""
        kp, vp = serving.widen(back(self.kp)), serving.widen(back(self.vp))
        embed, inv = back(self.embed), back(self.inv)
        step = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
        for r, ids in enumerate(tokens):
            x = embed[np.asarray(ids, int)]
            k = serving.rope(x[:, self.hq:self.hq + self.hkv], np.arange(len(ids)), inv)
            at = np.arange(len(ids))
            page = self.table_host[r][at // PS]
            assert (np.abs(kp[page, :, at % PS] - k) <= step * np.abs(k) + 2.0 ** -20 * np.abs(serving.widen(x)).max()).all()
            assert (vp[page, :, at % PS] == serving.widen(x[:, self.hq + self.hkv:])).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[37, 1, 300], [1], [16, 15, 17, 600, 2]])
def test_prompt_then_tokens(ada, dtype, lens):
    import torch
    s = Server(ada, sum(lens), lens, dtype)
    rng = np.random.default_rng(1)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    tokens = [back(s.prompt)[a:b].tolist() for a, b in zip(s.indptr_host, s.indptr_host[1:])]
    now = np.array(lens)
    with torch.cuda.stream(stream):
        for n in range(6):
            s.u.copy_(torch.from_numpy(rng.random(s.B).astype(np.float32)))
            print("serving step", n, "lengths", now.tolist(), flush=True)
            if n == 0:
                s.prefill()
            else:
                for r, t in enumerate(back(s.token)):
                    tokens[r].append(int(t))
                now = now + 1
                s.step()
            stream.synchronize()
            s.check(s.indptr_host if n == 0 else np.arange(s.B + 1), now)
    s.stored(tokens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_from_a_graph(ada, dtype):
    """The step of one token captured and replayed gives what the eager step
    gives, token by token, cache and all, with eager steps in between."""
    import torch
    lens = [37, 1, 300, 64]
    a, b = Server(ada, 5, lens, dtype), Server(ada, 5, lens, dtype)
    rng = np.random.default_rng(2)
    a.prefill()
    b.prefill()
    keep = a.lens.clone(), a.token.clone(), a.kp.clone(), a.vp.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.step()
    for dst, src in zip((a.lens, a.token, a.kp, a.vp), keep):
        dst.copy_(src)
    torch.cuda.synchronize()
    for n in range(6):
        u = torch.from_numpy(rng.random(len(lens)).astype(np.float32))
        a.u.copy_(u)
        b.u.copy_(u)
        torch.cuda.synchronize()
        print("graph step", n, flush=True)
        g.replay()
        b.step()
        torch.cuda.synchronize()
        for x, y in ((a.token, b.token), (a.lens, b.lens), (a.out, b.out), (a.kp, b.kp), (a.vp, b.vp)):
            assert back(x).tobytes() == back(y).tobytes()
        a.check(np.arange(len(lens) + 1), np.array(lens) + n + 1)


def test_two_servers_on_two_streams(ada):
    """Two batches served at once on two streams, each with workspaces of its own, as one after the other."""
    import torch
    lens = [[500, 3, 64], [129, 700]]
    alone = [Server(ada, 7 + i, x, "bf16") for i, x in enumerate(lens)]
    both = [Server(ada, 7 + i, x, "bf16") for i, x in enumerate(lens)]
    for s in alone:
        s.prefill()
        for _ in range(5):
            s.step()
        torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for x in streams:
        x.wait_stream(torch.cuda.current_stream())
    for n in range(6):
        for s, x in zip(both, streams):
            with torch.cuda.stream(x):
                s.step() if n else s.prefill()
    torch.cuda.synchronize()
    for s, t in zip(alone, both):
        for x, y in ((s.token, t.token), (s.lens, t.lens), (s.out, t.out), (s.kp, t.kp), (s.vp, t.vp)):
            assert back(x).tobytes() == back(y).tobytes()


@pytest.mark.parametrize("new,ctx", [([100], [4000]), ([600, 40], [600, 40])])
def test_prompt_attention_from_a_graph(ada, new, ctx):
    """Split keys (a workspace) and whole ones, replayed with new queries and eager work in between."""
    import torch
    rng = np.random.default_rng(9)
    hq, hkv, d = 8, 2, 128
    indptr, ctx = np.concatenate([[0], np.cumsum(new)]).astype(np.int32), np.asarray(ctx, np.int32)
    c = Cache(rng, ctx, hkv, d, "bf16")
    kp, vp, table, ip, cl = (to_dev(x) for x in (c.k, c.v, c.table, indptr, ctx))
    need = ada.adaserve_prompt_attn_workspace_bytes(indptr, ctx, hq, hkv, d, PS, ada.ADASERVE_BF16)
    assert (need > 0) == (new == [100])
    q = to_dev(typed(rng.standard_normal((int(indptr[-1]), hq, d)), "bf16"))

    def call(out, ws):
        ada.adaserve_prompt_attn(token_indptr=ip, token_indptr_host=indptr, q=q, k_pages=kp, v_pages=vp, block_table=table,
                                 context_len=cl, context_len_host=ctx, sm_scale=d ** -0.5, out=out, workspace=ws)
    ws = [torch.full((max(need, 1),), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    out, eager = torch.empty_like(q), torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, ws[0])
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(out, ws[0])
    for n in range(3):
        x = typed(rng.standard_normal(tuple(q.shape)), "bf16")
        q.copy_(to_dev(x))
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        call(eager, ws[1])
        torch.cuda.synchronize()
        assert back(out).tobytes() == back(eager).tobytes()
    ref, size, reach = serving.paged_attention(x, indptr, c.k, c.v, c.table, ctx, d ** -0.5)
    err = np.abs(serving.widen(back(out)) - ref)
    assert (err <= attention_bound("bf16", ref, size, reach, int(ctx.max()), d)).all()


def test_stream_given_by_the_caller(ada):
    """`stream=` puts the work on that stream, behind what waits there."""
    import torch
    s = Server(ada, 15, [200, 9], "bf16")
    s.prefill()
    s.step()
    torch.cuda.synchronize()
    out, token = torch.zeros_like(s.out), torch.full_like(s.token, -7)
    side = torch.cuda.Stream()
    q = torch.zeros_like(s.q)
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)   # about a millisecond
        q.copy_(s.q)
    ada.adaserve_decode_attn(q=q, k_pages=s.kp, v_pages=s.vp, block_table=s.table, context_len=s.lens, max_context=s.most,
                             sm_scale=s.scale, out=out, workspace=s.ws_decode, stream=side)
    ada.adaserve_sample(logits=out.reshape(s.B, -1), vocab=s.vocab, u=s.u, out_token=token, workspace=s.ws_sample, stream=side,
                        **s.par_dev)
    side.synchronize()
    assert back(out).tobytes() == back(s.out).tobytes() and token.tolist() == s.token.tolist()
