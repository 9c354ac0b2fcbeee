"""Tables kept on the GPU, summaries, selection and attention over selected blocks as a program runs them: a step captured in a graph and replayed with other
lengths, draft trees whose accepted path becomes context, contexts on two streams, pools beyond 2^31 elements."""
import numpy as np
import pytest
import torch

from tests.block_refs import assign, mask_words, masked_attention, positions, random_lists, random_trees, select, summary
from tests.operator_refs import F8, PAGE, Paged, context, cuda

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _attention_of(q, k, v, lists, bt, ctx, block, b, n, scale, own=None, vis=None):
    """(out, bound) of sequence b's n rows q [n, Hq, D]; own: the tree's keys and values."""
    hkv, d = k.shape[2:]
    G = q.shape[1] // hkv
    outs = []
    for h in range(hkv):
        seen = positions(lists[h][lists[h] >= 0], ctx, block)
        pos = seen if own is not None else np.concatenate([seen, ctx + np.arange(n)])
        at = cuda(bt[b, pos // PAGE] * PAGE + pos % PAGE, torch.int64)
        kk, vv = k.view(-1, hkv, d)[at, h], v.view(-1, hkv, d)[at, h]
        if own is not None:
            kk, vv = torch.cat((kk, own[0][:n, h])), torch.cat((vv, own[1][:n, h]))
            seen_by = np.concatenate([np.ones((n, len(pos)), bool), vis[:n, :n]], 1)
        else:
            seen_by = pos[None] <= (ctx + np.arange(n))[:, None]
        outs.append(masked_attention(q[:, h * G:h * G + G], kk, vv, cuda(seen_by, torch.bool), scale))
    return tuple(torch.cat([o[i] for o in outs], 1) for i in (0, 2))


@pytest.mark.parametrize("hq,hkv,d,block,K", [(16, 4, 64, 32, 6), (8, 8, 128, 64, 3), (32, 2, 128, 16, 9)])
def test_a_step_captured_and_replayed(hq, hkv, d, block, K):
    B, N, pages, width = 3, 160, 400, 120
    rng = np.random.default_rng(hq)
    g = torch.Generator(device="cuda").manual_seed(hq)
    cb = context(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d)
    free = rng.permutation(pages)
    table, held, n_free = np.full((B, width), -1), np.zeros(B, np.int64), pages
    dev = dict(table=cuda(table), held=cuda(held), free=cuda(free), n_free=cuda([pages]), start=cuda(np.zeros(B + 1)), ctx=cuda(np.zeros(B)), to=cuda(np.zeros(B)))
    k_pool, v_pool = (torch.full((pages, PAGE, hkv, d), float("nan"), device="cuda", dtype=BF) for _ in range(2))      # as an allocator leaves it
    mean, scale = cb.alloc_summary(pages)
    x = torch.zeros(N, hq + 2 * hkv, d, device="cuda", dtype=BF)
    q = torch.zeros(N, hq, d, device="cuda", dtype=BF)
    out, blocks = torch.zeros_like(q), torch.zeros(B, hkv, K, device="cuda", dtype=torch.int32)
    slots = dict(slots=torch.zeros(N, device="cuda", dtype=torch.int64), positions=torch.zeros(N, device="cuda", dtype=torch.int32), seqs=torch.zeros(N, device="cuda", dtype=torch.int32))

    def step():
        cb.cb_pages_assign(dev["to"], dev["table"], dev["held"], dev["free"], dev["n_free"])
        cb.cb_slot_map(dev["start"], dev["ctx"], dev["table"], pages, N, res=slots)
        cb.cb_chunk_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], dev["start"], dev["ctx"], k_pool, v_pool, dev["table"], q_out=q)
        cb.cb_block_summary(k_pool, dev["table"], dev["ctx"], dev["to"], mean, scale, block=block)
        cb.cb_block_select(q, mean, scale, dev["table"], dev["ctx"], q_start=dev["start"], block=block, n_select=K, n_first=1, n_last=2, max_chunk=60, max_ctx=1900, blocks=blocks)
        cb.cb_block_attn(q, k_pool, v_pool, dev["table"], dev["start"], dev["ctx"], blocks, block=block, out=out, max_chunk=60, max_ctx=1920)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    ctx = np.zeros(B, np.int64)
    for turn in range(14):
        new = np.array([1, 1, 1]) if turn % 3 == 2 else rng.integers(0, 31, B) + (0 if turn else 20)
        if turn == 7:                                                        # one sequence is finished, another takes its place
            ctx[1], new[1] = 0, 25
        if turn == 9:
            new = np.zeros(B, np.int64)
        s = np.concatenate([[0], np.cumsum(new)])
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        if turn == 7:
            dev["to"].copy_(cuda(np.where(np.arange(B) == 1, 0, ctx)))
            cb.cb_pages_assign(dev["to"], dev["table"], dev["held"], dev["free"], dev["n_free"])
            n_free, _ = assign(np.where(np.arange(B) == 1, 0, ctx), table, held, free, n_free)
        for name, v in (("start", s), ("ctx", ctx), ("to", ctx + new)):
            dev[name].copy_(cuda(v))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert cb.cb_poll_status()[0] == 0
        n_free, alone = assign(ctx + new, table, held, free, n_free)
        assert not alone and np.array_equal(dev["table"].cpu().numpy(), table) and np.array_equal(dev["free"].cpu().numpy(), free) and int(dev["n_free"]) == n_free
        got = blocks.cpu().numpy()
        assert bool((out[s[-1]:] == 7).all()) and bool((slots["seqs"][s[-1]:] == -1).all())
        for b in range(B):
            rows = slice(s[b], s[b + 1])
            pos = ctx[b] + np.arange(new[b])
            at = cuda(table[b, pos // PAGE] * PAGE + pos % PAGE, torch.int64)
            assert torch.equal(slots["slots"][rows], at) and slots["positions"][rows].tolist() == pos.tolist()
            assert torch.equal(k_pool.view(-1, hkv, d)[at], x[rows, hq:hq + hkv]) and torch.equal(v_pool.view(-1, hkv, d)[at], x[rows, hq + hkv:])
            nb = -(-int(ctx[b]) // block)
            first = cuda(table[b, np.arange(nb) * block // PAGE], torch.int64)
            for h in range(hkv):
                want = select(q[rows, h * (hq // hkv):(h + 1) * (hq // hkv)].reshape(-1, d), mean[first, h], scale[first, h], K, 1, 2)
                assert got[b, h].tolist() == want + [-1] * (K - len(want))
            for j in range(int(ctx[b]) // block, -(-int(ctx[b] + new[b]) // block)):
                t = np.arange(j * block, min((j + 1) * block, ctx[b] + new[b]))
                m, _ = summary(k_pool.view(-1, hkv, d)[cuda(table[b, t // PAGE] * PAGE + t % PAGE, torch.int64)])
                assert torch.equal(mean[table[b, j * block // PAGE]].long(), m)
            if new[b]:
                ref, bound = _attention_of(q[rows], k_pool, v_pool, got[b], table, int(ctx[b]), block, b, int(new[b]), d ** -0.5)
                assert bool(((out[rows].to(F8) - ref).abs() <= bound).all()), (turn, b)
        ctx = ctx + new


def test_trees_whose_accepted_path_becomes_context():
    B, T, hq, hkv, d, block, K = 3, 40, 16, 4, 64, 32, 5
    rng = np.random.default_rng(3)
    c = Paged([60] * B, [700, 31, 290], hkv, d, seed=3)                      # room for 60 tokens behind each
    cb = context(batch=B, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_nodes=T, max_depth=6)
    mean, scale = cb.alloc_summary(c.num_pages)
    ctx_d = c.d_ctx.clone()
    cb.cb_block_summary(c.k, c.block_table, cuda(np.zeros(B)), ctx_d, mean, scale, block=block)
    ctx = c.ctx.copy()
    for turn in range(4):
        n = rng.integers(1, T + 1, B)
        vis, words = random_trees(B, T, n, turn)
        q, kt, vt = (torch.randn(B, T, h, d, generator=c.g, device="cuda").to(BF) for h in (hq, hkv, hkv))
        blocks = cb.cb_block_select(q, mean, scale, c.block_table, ctx_d, n_nodes=cuda(n), block=block, n_select=K)
        out = cb.cb_block_tree_attn(q, c.k, c.v, c.block_table, ctx_d, kt, vt, words, cuda(n), blocks, block=block)
        lists = blocks.cpu().numpy()
        for b in range(B):
            m = int(n[b])
            nb = -(-int(ctx[b]) // block)
            first = cuda(c.bt[b, np.arange(nb) * block // PAGE], torch.int64)
            for h in range(hkv):
                want = select(q[b, :m, h * 4:h * 4 + 4].reshape(-1, d), mean[first, h], scale[first, h], K, 1, 2)
                assert lists[b, h].tolist() == want + [-1] * (K - len(want))
            ref, bound = _attention_of(q[b, :m], c.k, c.v, lists[b], c.bt, int(ctx[b]), block, b, m, d ** -0.5, own=(kt[b], vt[b]), vis=vis[b])
            assert bool(((out[b, :m].to(F8) - ref).abs() <= bound).all()), (turn, b)
        # the longest path below the root that the mask has, accepted
        acc, nodes = [], np.full((B, 6), -1)
        for b in range(B):
            deep = max(range(int(n[b])), key=lambda i: (min(vis[b, i].sum(), 7), -i))
            path = np.nonzero(vis[b, deep])[0][1:7]
            nodes[b, :len(path)] = path
            acc.append(len(path))
        old = ctx_d.clone()
        cb.cb_kv_commit(c.k, c.v, c.block_table, ctx_d, kt, vt, cuda(acc), cuda(nodes))
        cb.cb_block_summary(c.k, c.block_table, old, ctx_d, mean, scale, block=block)
        ctx = ctx + 1 + np.array(acc)
        assert ctx_d.tolist() == ctx.tolist() and cb.cb_poll_status()[0] == 0


def test_two_contexts_on_two_streams():
    jobs = []
    for k, (hq, hkv, d, new, ctx) in enumerate([(32, 8, 128, [1] * 40, list(range(50, 8050, 200))), (64, 8, 64, [30, 1, 40, 7], [1000, 2000, 0, 9000])]):
        c = Paged(new, ctx, hkv, d, seed=k)
        q = (torch.randn(int(c.q_start[-1]), hq, d, generator=c.g, device="cuda") * 1.5).to(BF)
        cb = context(batch=len(new), n_q_heads=hq, n_kv_heads=hkv, head_dim=d)
        mean, scale = cb.alloc_summary(c.num_pages)
        res = [(torch.zeros(len(new), hkv, 9, device="cuda", dtype=torch.int32), torch.empty_like(q)) for _ in range(6)]
        jobs.append((c, q, cb, mean, scale, torch.cuda.Stream(), res))
    torch.cuda.synchronize()
    for k in range(6):
        for c, q, cb, mean, scale, st, res in jobs:
            cb.cb_block_summary(c.k, c.block_table, cuda(0 * c.ctx) if k == 0 else c.d_ctx, c.d_ctx, mean, scale, stream=st)
            cb.cb_block_select(q, mean, scale, c.block_table, c.d_ctx, q_start=c.d_start, n_select=9, max_chunk=int(c.new.max()), blocks=res[k][0], stream=st)
            cb.cb_block_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, res[k][0], out=res[k][1], max_chunk=int(c.new.max()), stream=st)
    torch.cuda.synchronize()
    for c, q, cb, mean, scale, st, res in jobs:
        assert cb.cb_poll_status()[0] == 0
        for k in range(1, 6):
            assert torch.equal(res[k][0], res[0][0]) and torch.equal(res[k][1], res[0][1])
        lists = res[0][0].cpu().numpy()
        for b in range(0, len(c.new), 3):
            rows = slice(c.q_start[b], c.q_start[b + 1])
            ref, bound = _attention_of(q[rows], c.k, c.v, lists[b], c.bt, int(c.ctx[b]), 64, b, int(c.new[b]), q.shape[2] ** -0.5)
            assert bool(((res[0][1][rows].to(F8) - ref).abs() <= bound).all()), b


def test_calls_in_a_row_without_a_pause():
    """Every kernel may be scheduled while the one before it ends: what one writes the next one reads, over and over."""
    c = Paged([1] * 9, [1000 + 37 * i for i in range(9)], 8, 128)
    q = torch.randn(9, 32, 128, generator=c.g, device="cuda").to(BF)
    cb = context(batch=9, n_q_heads=32, n_kv_heads=8, head_dim=128)
    mean, scale = cb.alloc_summary(c.num_pages)
    zero, outs = cuda(np.zeros(9)), []
    for k in range(40):
        c.k.mul_(-1.0)                                                       # the blocks' order turns round
        cb.cb_block_summary(c.k, c.block_table, zero, c.d_ctx, mean, scale)
        blocks = cb.cb_block_select(q, mean, scale, c.block_table, c.d_ctx, q_start=c.d_start, n_select=5, max_chunk=1)
        outs.append((blocks, cb.cb_block_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, blocks, max_chunk=1)))
    for k in range(2, 40):
        assert torch.equal(outs[k][0], outs[k & 1][0]) and torch.equal(outs[k][1], outs[k & 1][1])
    assert not torch.equal(outs[0][0], outs[1][0]) and cb.cb_poll_status()[0] == 0


def test_pools_beyond_32_bits():
    """Pages whose first element lies 2^31 elements and more into the pool."""
    pages, hkv, d = (1 << 17) + 64, 8, 128
    pool = torch.zeros(pages, PAGE, hkv, d, device="cuda", dtype=BF)         # keys and values at once
    c = Paged([1, 20], [900, 130], hkv, d, seed=1)
    far = pages - c.num_pages + c.bt
    at = cuda(np.arange(pages - c.num_pages, pages), torch.int64)
    pool[at] = c.k
    c.k = c.v = pool
    c.bt, c.block_table = far, cuda(far)
    q = torch.randn(21, 32, d, generator=c.g, device="cuda").to(BF)
    cb = context(batch=2, n_q_heads=32, n_kv_heads=hkv, head_dim=d)
    mean, scale = cb.alloc_summary(pages)
    cb.cb_block_summary(pool, c.block_table, cuda([0, 0]), c.d_ctx, mean, scale)
    blocks = cb.cb_block_select(q, mean, scale, c.block_table, c.d_ctx, q_start=c.d_start, n_select=4)
    lists = blocks.cpu().numpy()
    for max_chunk in (0, 20):
        out = cb.cb_block_attn(q, pool, pool, c.block_table, c.d_start, c.d_ctx, blocks, max_chunk=max_chunk)
        for b in range(2):
            rows = slice(c.q_start[b], c.q_start[b + 1])
            nb = -(-int(c.ctx[b]) // 64)
            first = cuda(far[b, np.arange(nb) * 4], torch.int64)
            for h in range(hkv):
                want = select(q[rows, h * 4:h * 4 + 4].reshape(-1, d), mean[first, h], scale[first, h], 4, 1, 2)
                assert lists[b, h].tolist() == want + [-1] * (4 - len(want))
            ref, bound = _attention_of(q[rows], pool, pool, lists[b], far, int(c.ctx[b]), 64, b, int(c.new[b]), d ** -0.5)
            assert bool(((out[rows].to(F8) - ref).abs() <= bound).all()), b
    one = context(batch=1, n_q_heads=32, n_kv_heads=hkv, head_dim=d)
    out = one.cb_block_attn(q[:1], pool, pool, c.block_table[:1], c.d_start[:2], c.d_ctx[:1], blocks[:1], max_chunk=1)
    ref, bound = _attention_of(q[:1], pool, pool, lists[0], far, 900, 64, 0, 1, d ** -0.5)
    assert bool(((out.to(F8) - ref).abs() <= bound).all()) and cb.cb_poll_status()[0] == 0


@pytest.mark.parametrize("new", [[1], [3]])
def test_a_context_of_long_lists(new):
    """Lists of 1,000 blocks: page numbers beyond the first 64 of a warp, and all blocks of 16."""
    c = Paged(new, [20000], 1, 64)
    q = torch.randn(new[0], 4, 64, generator=c.g, device="cuda").to(BF)
    cb = context(n_q_heads=4, n_kv_heads=1)
    lists = random_lists(c.ctx, 1, 1000, 16, seed=0)
    out = cb.cb_block_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, cuda(lists), block=16, max_chunk=new[0])
    ref, bound = _attention_of(q, c.k, c.v, lists[0], c.bt, 20000, 16, 0, new[0], 0.125)
    assert bool(((out.to(F8) - ref).abs() <= bound).all())
    lists = random_lists(c.ctx, 1, 100, 128, seed=0)                         # many units: no cluster shares them, a warp has hundreds of pages
    many = Paged([1] * 160, [13000] * 160, 1, 64, seed=2)
    qm = torch.randn(160, 4, 64, generator=many.g, device="cuda").to(BF)
    lists = random_lists(many.ctx, 1, 100, 128, seed=0)
    cbm = context(batch=160, n_q_heads=4, n_kv_heads=1)
    out = cbm.cb_block_attn(qm, many.k, many.v, many.block_table, many.d_start, many.d_ctx, cuda(lists), block=128, max_chunk=1)
    for b in (0, 77, 159):
        ref, bound = _attention_of(qm[b:b + 1], many.k, many.v, lists[b], many.bt, 13000, 128, b, 1, 0.125)
        assert bool(((out[b:b + 1].to(F8) - ref).abs() <= bound).all())
