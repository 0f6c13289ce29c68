"""The serving operators together, as a decoding program uses them: projection,
append, attention, output projection, lm_head, sample; eagerly, captured in a
graph that is replayed with new contents, and on a stream of their own."""

import sys

import pytest
import torch

import serving
from serving import DEV
from paper_2608_28003_amd import w8a8

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

D, HEADS, VOCAB = 1152, 4, 8192


class Model:
    """One attention layer and a small lm_head, INT8 weights."""

    def __init__(self):
        g = serving.gen(1)
        w = lambda n, k: (torch.randn((n, k), generator=g) * 0.03).to(torch.bfloat16).to(DEV)
        self.qkv = w8a8.LinearW8A8.from_weight(w((HEADS + 2) * 256, D))
        self.o = w8a8.LinearW8A8.from_weight(w(D, HEADS * 256))
        self.head = w8a8.LinearW8A8.from_weight(w(VOCAB, D))
        self.embed = (torch.randn((VOCAB, D), generator=g)).to(torch.bfloat16).to(DEV)
        self.rope = w8a8.Rope.make(256, theta=1e6, scaling="linear", factor=8.0)

    def step(self, tokens, cache, batch, u, window, stream=None):
        x = self.embed[tokens]
        qkv = w8a8.linear(self.qkv, x, out_dtype=torch.bfloat16, stream=stream)
        q = w8a8.kv_append(qkv, cache, batch, HEADS, rope=self.rope, stream=stream)
        a = w8a8.attn_paged(q, cache, batch, window=window, stream=stream)
        y = x + w8a8.linear(self.o, a.view(a.shape[0], -1), out_dtype=torch.bfloat16, stream=stream)
        logits = w8a8.lm_head(self.head, w8a8.rmsnorm(y.contiguous(), stream=stream), stream=stream)
        return w8a8.sample(logits[batch.q_start[1:].long() - 1].contiguous(), u, 0.8, 50, 0.95, 0.01, stream=stream)


def batch_of(table, fresh, ctx):
    start = torch.tensor([0] + fresh, dtype=torch.int32).cumsum(0, dtype=torch.int32).to(DEV)
    return w8a8.PagedBatch(table, start, torch.tensor(ctx, dtype=torch.int32, device=DEV), max(fresh))


@pytest.mark.parametrize("int8", [True, False])
def test_prompts_in_chunks_then_tokens(int8):
    """Three prompts of different lengths: at once, or in two chunks, or token by
    token, the cache and the attention of the last token come out the same up to
    the sums' order; the decode steps after it draw tokens."""
    m, page = Model(), 16
    lens = [37, 64, 5]
    g = serving.gen(7)
    prompts = [torch.randint(0, VOCAB, (n,), generator=g).to(DEV) for n in lens]
    table = torch.randperm(3 * 8, generator=g).int().view(3, 8).to(DEV)

    def feed(parts):
        cache = w8a8.PagedKV.empty(24, page, int8=int8)
        done = [0, 0, 0]
        for part in parts:
            fresh = [min(part, n - d) for n, d in zip(lens, done)]
            ids = torch.cat([p[d:d + f] for p, d, f in zip(prompts, done, fresh)])
            done = [d + f for d, f in zip(done, fresh)]
            b = batch_of(table, fresh, done)
            qkv = w8a8.linear(m.qkv, m.embed[ids], out_dtype=torch.bfloat16)
            q = w8a8.kv_append(qkv, cache, b, HEADS, rope=m.rope)
            a = w8a8.attn_paged(q, cache, b, window=50)
        return cache, a[-1]

    whole, last = feed([64])
    for parts in ([32, 32], [1] * 64):
        cache, a = feed(parts)
        for t, r in zip((cache.k, cache.v, cache.sk, cache.sv) if int8 else (cache.k, cache.v),
                        (whole.k, whole.v, whole.sk, whole.sv) if int8 else (whole.k, whole.v)):
            assert torch.equal(t, r)  # rows do not depend on how the prompt is cut
    # the second prompt's last token came last in every feed but the whole one's, where the third's did
    u = torch.rand((12, 3), generator=g).to(DEV)
    ctx, tokens, drawn = list(lens), torch.stack([p[-1] for p in prompts]), []
    for i in range(12):
        ctx = [c + 1 for c in ctx]
        tokens, prob = m.step(tokens, whole, batch_of(table, [1, 1, 1], ctx), u[i], 50)
        assert ((tokens >= 0) & (tokens < VOCAB)).all() and (prob > 0).all()
        drawn.append(tokens)
    assert len(torch.stack(drawn).unique()) > 3


def test_graph_replays_follow_their_inputs():
    """A captured step replayed with new tokens, lengths, tables and uniform
    numbers gives what the eager step gives; two graphs share no state."""
    m = Model()
    g = serving.gen(9)
    caches = [w8a8.PagedKV.empty(40, 16) for _ in range(2)]
    table = torch.randperm(40, generator=g).int().view(2, 20).to(DEV)
    tokens, u = torch.zeros(2, dtype=torch.int64, device=DEV), torch.zeros(2, device=DEV)
    b = batch_of(table.clone(), [1, 1], [1, 1])
    ws = torch.empty(max(1, w8a8.attn_paged_workspace_bytes(2, HEADS, 1, 256, 2, 1, 320)), dtype=torch.uint8, device=DEV)
    sws = torch.empty(max(1, w8a8.sample_workspace_bytes(2, VOCAB, torch.bfloat16)), dtype=torch.uint8, device=DEV)

    def step(cache):
        x = m.embed[tokens]
        q = w8a8.kv_append(w8a8.linear(m.qkv, x, out_dtype=torch.bfloat16), cache, b, HEADS, rope=m.rope)
        a = w8a8.attn_paged(q, cache, b, ws=ws)
        y = w8a8.linear(m.o, a.view(2, -1), out_dtype=torch.bfloat16)
        return a, *w8a8.sample(w8a8.lm_head(m.head, y), u, 0.9, 40, 0.9, ws=sws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[0])
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):  # two graphs over the same workspaces
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs = step(caches[0])
        graphs.append((gr, outs))
    for t in (caches[0].k, caches[0].v, caches[0].sk, caches[0].sv):
        t.zero_()
    for i in range(8):
        tokens.copy_(torch.randint(0, VOCAB, (2,), generator=g))
        u.copy_(torch.rand(2, generator=g))
        b.ctx_len.copy_(torch.tensor([1 + 30 * i, 5 + 20 * i]))
        b.table.copy_(table.flip(0) if i % 2 else table)
        want = step(caches[1])
        torch.cuda.synchronize()
        gr, outs = graphs[i % 2]
        gr.replay()
        torch.cuda.synchronize()
        for a, w in zip(outs, want):
            assert torch.equal(a, w), i
        assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].sv, caches[1].sv)


def test_a_stream_of_its_own():
    """Calls given a stream run there, with the memory they allocate."""
    h = serving.Paged([40, 1], [400, 300], 1, 256, 16, True, seed=4)
    cache, b = h.cache(w8a8), h.batch(w8a8)
    qkv = torch.randn((41, 1536), generator=serving.gen(5)).to(torch.bfloat16).to(DEV)
    r = w8a8.Rope.make(256)
    logits = (torch.randn((41, 9000), generator=serving.gen(6)) * 3).to(DEV)
    u = torch.rand(41, generator=serving.gen(7)).to(DEV)

    def calls(stream=None):
        q = w8a8.kv_append(qkv, cache, b, 4, rope=r, stream=stream)
        a = w8a8.attn_paged(q, cache, b, stream=stream)
        t, p = w8a8.sample(logits, u, top_p=0.9, stream=stream)
        k, v = w8a8.kv_read(cache, b, 41, stream=stream)
        return [q, a, t, p, k, v, w8a8.rope(r, q, b.ctx_len.new_zeros(41), stream=stream)]

    want = calls()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        got = calls(s)
        s.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert torch.cuda.current_stream() != s


@pytest.mark.parametrize("int8", [True, False])
def test_prompts_captured_and_replayed(int8):
    """Append and attention captured for up to 96 rows of four sequences, replayed
    with other lengths: prompts beside single tokens, single tokens only, one long
    sequence, none at all; against the eager calls, rows behind the last sequence untouched."""
    m, rows = Model(), 96
    g = serving.gen(11)
    caches = [w8a8.PagedKV.empty(4 * 70, 16, int8=int8) for _ in range(2)]
    table = torch.randperm(4 * 70, generator=g).int().view(4, 70).to(DEV)
    b = w8a8.PagedBatch(table, torch.zeros(5, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV), 90)
    qkv = torch.zeros((rows, (HEADS + 2) * 256), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(w8a8.attn_paged_workspace_bytes(rows, HEADS, 1, 256, 4, 90, 70 * 16), dtype=torch.uint8, device=DEV)
    q, out = (torch.zeros((rows, HEADS, 256), dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def step(cache, q, out):
        w8a8.kv_append(qkv, cache, b, HEADS, rope=m.rope, out=q)
        w8a8.attn_paged(q, cache, b, out=out, ws=ws)

    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        step(caches[0], q, out)
    done = [0, 0, 0, 0]
    for fresh in ([40, 1, 0, 20], [1, 1, 1, 1], [0, 90, 0, 0], [0, 0, 0, 0], [17, 16, 33, 30], [1, 0, 70, 2]):
        done = [d + f for d, f in zip(done, fresh)]
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        b.q_start.copy_(torch.tensor([0] + fresh).cumsum(0))
        b.ctx_len.copy_(torch.tensor(done))
        q.fill_(3.0)
        out.fill_(3.0)
        want_q, want = torch.full_like(q, 3.0), torch.full_like(out, 3.0)
        step(caches[1], want_q, want)
        torch.cuda.synchronize()
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, want_q) and torch.equal(out, want), fresh
        assert (out[sum(fresh):] == 3.0).all()
        assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)
