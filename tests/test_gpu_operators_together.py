"""The operators beside the step as programs run them at once: two contexts on two streams, and a whole layer's calls captured in a graph and
replayed with other lengths."""
import numpy as np
import pytest
import torch

from tests.operator_refs import F8, Paged, attention, context, cuda, likelihoods, normed_and_turned, rope_table

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_two_contexts_on_two_streams():
    """Each context has its own scratch: what one launch leaves half merged is nobody else's."""
    jobs = []
    for k, (hq, hkv, d, new, ctx) in enumerate([(32, 8, 128, [1] * 40, list(range(50, 4050, 100))), (8, 8, 64, [300, 1, 40, 7], [100, 2000, 0, 900])]):
        c = Paged(new, ctx, hkv, d, seed=k)
        q = (torch.randn(int(c.q_start[-1]), hq, d, generator=c.g, device="cuda") * 1.5).to(BF)
        cb = context(batch=len(new), n_q_heads=hq, n_kv_heads=hkv, head_dim=d, vocab=50000)
        outs = [(torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")) for _ in range(6)]
        x = torch.randn(30, 50000, generator=c.g, device="cuda")
        tok = torch.randint(50000, (30,), generator=c.g, device="cuda", dtype=torch.int32)
        jobs.append((c, q, cb, outs, torch.cuda.Stream(), x, tok, [cb._alloc_logprobs((30,), 9) for _ in range(6)]))
    torch.cuda.synchronize()
    for k in range(6):
        for c, q, cb, outs, st, x, tok, res in jobs:
            cb.cb_chunk_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, out=outs[k][0], lse=outs[k][1], max_chunk=int(c.new.max()), stream=st)
            cb.cb_logprobs(x, tok, top_k=9, res=res[k], stream=st)
    torch.cuda.synchronize()
    for c, q, cb, outs, st, x, tok, res in jobs:
        assert cb.cb_poll_status()[0] == 0
        hkv, d = c.k.shape[2:]
        for k in range(1, 6):
            assert torch.equal(outs[k][0], outs[0][0]) and torch.equal(outs[k][1], outs[0][1])
            assert all(torch.equal(res[k][n], res[0][n]) for n in res[0])
        for b in range(0, len(c.new), 3):
            lo, hi = c.q_start[b], c.q_start[b + 1]
            at = c.slots(b, 0, c.ctx[b] + c.new[b])
            ref, _, bound, _ = attention(q[lo:hi], c.k.view(-1, hkv, d)[at], c.v.view(-1, hkv, d)[at], int(c.ctx[b]), d ** -0.5)
            assert bool(((outs[0][0][lo:hi].to(F8) - ref).abs() <= bound).all()), b
        ref, bound = likelihoods(x, tok, 9)
        assert torch.equal(res[0]["top_ids"].long(), ref["top_ids"])
        assert all(bool(((res[0][n].to(F8) - ref[n]).abs() <= bound[n]).all()) for n in bound)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (16, 16, 128)])
def test_a_layer_captured_and_replayed(hq, hkv, d):
    """Append, attention and log probabilities in one graph; every replay has other projections, lengths and logits."""
    B, N, V = 3, 64, 5000
    rng = np.random.default_rng(hq)
    g = torch.Generator(device="cuda").manual_seed(hq)
    c = Paged([40] * B, [500] * B, hkv, d)
    table, w = rope_table(700, d), torch.ones(d, device="cuda", dtype=BF)
    x = torch.empty(N, hq + 2 * hkv, d, device="cuda", dtype=BF)
    logits, tok = torch.empty(N, V, device="cuda", dtype=BF), torch.zeros(N, device="cuda", dtype=torch.int32)
    start, ctx = cuda(np.zeros(B + 1)), cuda(np.zeros(B))
    q, out = torch.zeros(N, hq, d, device="cuda", dtype=BF), torch.zeros(N, hq, d, device="cuda", dtype=BF)
    lse = torch.zeros(N, hq, device="cuda")
    cb = context(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, vocab=V)
    res = cb._alloc_logprobs((N,), 4)

    def layer():
        cb.cb_chunk_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], start, ctx, c.k, c.v, c.block_table, rope=table, q_norm=w, k_norm=w, q_out=q)
        cb.cb_chunk_attn(q, c.k, c.v, c.block_table, start, ctx, out=out, lse=lse, max_chunk=40, max_ctx=560)
        cb.cb_logprobs(logits, tok, top_k=4, res=res)
    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for _ in range(5):
        new, old = rng.integers(0, 22, B), rng.integers(0, 500, B)
        s = np.concatenate([[0], np.cumsum(new)])
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        logits.copy_(torch.randn(logits.shape, generator=g, device="cuda") * 3)
        toks = rng.integers(0, V, N)
        toks[s[-1]:] = -1
        tok.copy_(cuda(toks))
        start.copy_(cuda(s))
        ctx.copy_(cuda(old))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert cb.cb_poll_status()[0] == 0
        assert (out[s[-1]:] == 7).all()
        for b in range(B):
            if new[b] == 0:
                continue
            rows, pos = slice(s[b], s[b + 1]), cuda(old[b] + np.arange(new[b]), torch.int64)
            z, bound = normed_and_turned(x[rows, :hq], w, 1e-6, table, pos, False)
            assert bool(((q[rows].to(F8) - z).abs() <= bound).all())
            at = c.slots(b, 0, old[b] + new[b])
            ref, _, bound, _ = attention(q[rows], c.k.view(-1, hkv, d)[at], c.v.view(-1, hkv, d)[at], int(old[b]), d ** -0.5)
            assert bool(((out[rows].to(F8) - ref).abs() <= bound).all()), b
        n = int(s[-1])
        if n:
            ref, bound = likelihoods(logits[:n], tok[:n], 4)
            assert torch.equal(res["top_ids"][:n].long(), ref["top_ids"])
            assert all(bool(((res[k][:n].to(F8) - ref[k]).abs() <= bound[k]).all()) for k in bound)
        assert (res["top_ids"][n:] == -1).all() and (res["logprobs"][n:] == 0).all()
