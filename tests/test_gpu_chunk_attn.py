"""cb_chunk_attn against causal attention in 64 bits: single tokens to long prompts, ragged batches, odd sizes, what lies behind the last token."""
import math

import numpy as np
import pytest
import torch

from tests.operator_refs import F8, PAGE, Paged, attention, context, cuda, normed_and_turned, rope_table

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _q(n, hq, d, g, scale=1.5):
    return (torch.randn(n, hq, d, generator=g, device="cuda") * scale).to(BF)


def _compare(out, lse, q, c, scale, seqs=None, k=None, v=None):
    hkv, d = c.k.shape[2:]
    k, v = (x.view(-1, hkv, d) for x in (c.k if k is None else k, c.v if v is None else v))
    for b in range(len(c.new)) if seqs is None else seqs:
        lo, hi = c.q_start[b], c.q_start[b + 1]
        if hi == lo:
            continue
        at = c.slots(b, 0, c.ctx[b] + c.new[b])
        ref, rl, b_out, b_lse = attention(q[lo:hi], k[at], v[at], int(c.ctx[b]), scale)
        off, loff = (out[lo:hi].to(F8) - ref).abs(), (lse[lo:hi].to(F8) - rl).abs()
        assert bool((off <= b_out).all()), (b, int(c.new[b]), int(c.ctx[b]), float((off - b_out).max()), float(off.max()))
        assert bool((loff <= b_lse).all()), (b, float((loff - b_lse).max()), float(loff.max()))


def _run(c, q, flags=0, hints=True, cb=None, scale=0.0, k=None, v=None, max_ctx=None, max_chunk=None):
    hkv, d = c.k.shape[2:]
    n, hq = q.shape[:2]
    cb = cb or context(batch=len(c.new), n_q_heads=hq, n_kv_heads=hkv, head_dim=d, flags=flags)
    out, lse = torch.full_like(q, 7.0), torch.full((n, hq), 7.0, device="cuda")
    cb.cb_chunk_attn(q, c.k if k is None else k, c.v if v is None else v, c.block_table, c.d_start, c.d_ctx, out=out, lse=lse,
                     max_chunk=(int(c.new.max()) if hints else 0) if max_chunk is None else max_chunk,
                     max_ctx=(int((c.new + c.ctx).max()) if hints else 0) if max_ctx is None else max_ctx, scale=scale)
    st, _ = cb.cb_poll_status()
    return out, lse, st


SHAPES = [
    # hq, hkv, d, new, ctx
    (8, 8, 64, [1], [0]),                                         # a sequence's first token
    (32, 32, 128, [1], [4096]),
    (32, 8, 128, [1] * 9, [0, 1, 127, 128, 129, 15, 16, 17, 2000]),
    (64, 8, 128, [1, 0, 1], [300, 77, 5000]),
    (28, 4, 128, [3, 18, 19, 36, 37], [0, 5, 250, 1, 128]),       # 18 tokens a row tile
    (5, 1, 64, [25, 26, 51, 1], [0, 100, 30, 3]),
    (48, 3, 64, [8, 9, 40], [7, 0, 300]),                         # 16 heads a group
    (8, 8, 128, [128, 127, 129, 256, 257, 1], [0, 0, 1, 3, 128, 129]),
    (16, 4, 64, [509, 0, 1, 64, 200, 33], [3, 9, 1203, 640, 0, 31]),
    (4, 2, 128, [700], [0]),
    (6, 2, 64, [1000, 1], [513, 0]),
    (2, 1, 128, [2], [9000]),
    (40, 40, 64, [15, 16, 17], [1, 0, 15]),
]


@pytest.mark.parametrize("hq,hkv,d,new,ctx", SHAPES)
@pytest.mark.parametrize("flags", [0, 2])
def test_shapes(hq, hkv, d, new, ctx, flags):
    c = Paged(new, ctx, hkv, d, seed=hq + len(new))
    q = _q(int(c.q_start[-1]), hq, d, c.g)
    for hints in (True, False):
        out, lse, st = _run(c, q, flags, hints)
        assert st == 0
        _compare(out, lse, q, c, d ** -0.5)


def test_many_sequences():
    """300 sequences, one token each among chunks: the search and the schedule over many."""
    rng = np.random.default_rng(2)
    new = np.where(rng.random(300) < 0.8, 1, rng.integers(0, 70, 300))
    ctx = rng.integers(0, 600, 300)
    c = Paged(new, ctx, 2, 64)
    q = _q(int(c.q_start[-1]), 8, 64, c.g)
    out, lse, st = _run(c, q)
    assert st == 0
    _compare(out, lse, q, c, 64 ** -0.5)


@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 128), (8, 8, 64), (32, 32, 128), (16, 2, 128), (64, 8, 64), (148, 148, 64)])
def test_single_tokens_of_small_batches_and_then_a_large_launch(hq, hkv, d):
    """Units shared by up to 32 CTAs, from one key to many tiles each; launches of few CTAs between launches of all (what is counted for the CTAs of
    one may not reach the next)."""
    c2 = Paged([90, 1, 33], [700, 2000, 5], hkv, d, seed=4)
    q2 = _q(int(c2.q_start[-1]), hq, d, c2.g)
    for new, ctx in (([1], [0]), ([1], [127]), ([1], [128]), ([1], [1300]), ([1], [5000]), ([1, 1], [300, 3]), ([1, 0, 1], [1000, 5, 129])):
        cb = context(batch=len(new), n_q_heads=hq, n_kv_heads=hkv, head_dim=d)
        c = Paged(new, ctx, hkv, d, seed=2)
        q = _q(int(c.q_start[-1]), hq, d, c.g)
        for _ in range(2):
            out, lse, st = _run(c, q, cb=cb)
            assert st == 0
            _compare(out, lse, q, c, d ** -0.5)
        if len(new) == 3:
            for _ in range(3):
                out, lse, st = _run(c2, q2, cb=cb)
                assert st == 0
                _compare(out, lse, q2, c2, d ** -0.5)
                out, lse, st = _run(c, q, cb=cb)
                _compare(out, lse, q, c, d ** -0.5)


@pytest.mark.parametrize("d", [64, 128])
def test_long_chunk_on_a_long_context(d):
    c = Paged([1500, 1, 2100], [6000, 9000, 0], 2, d)
    q = _q(int(c.q_start[-1]), 8, d, c.g)
    out, lse, st = _run(c, q)
    assert st == 0
    _compare(out, lse, q, c, d ** -0.5)


@pytest.mark.parametrize("flags", [0, 2])
@pytest.mark.parametrize("d,hkv,new,ctx", [(64, 1, [70], [900]), (128, 1, [70], [900]), (64, 2, [1, 1, 1], [1500, 300, 129]), (128, 4, [1, 1], [2000, 700]),
                                           (64, 3, [300, 1, 200], [0, 800, 130]), (128, 2, [257, 33], [128, 500])])
def test_scores_far_apart_and_rising(d, hkv, new, ctx, flags):
    """A row's maximum comes late, by far: every reference is passed again and again.  Two row tiles, single tokens (shared by CTAs, or two heads at a
    time), and both mixed."""
    c = Paged(new, ctx, hkv, d)
    for b in range(len(new)):
        at = c.slots(b, 0, ctx[b] + new[b])
        step = torch.linspace(0.1, 30, len(at), device="cuda")
        c.k.view(-1, hkv, d)[at] = step[:, None, None].to(BF).expand(-1, hkv, d).contiguous()
    q = torch.ones(int(c.q_start[-1]), 2 * hkv, d, device="cuda", dtype=BF)
    q[::2] = -1.0
    q[:, 1::3] *= 0.25
    for hints in (True, False):
        for scale in (0.0, 1.0):
            out, lse, st = _run(c, q, flags, hints, scale=scale)
            assert st == 0
            _compare(out, lse, q, c, scale or d ** -0.5)


@pytest.mark.parametrize("flags", [0, 2])
@pytest.mark.parametrize("hq,hkv,d,new,ctx", [(8, 2, 64, [1, 1, 1], [0, 20, 143]), (4, 4, 128, [37, 1, 150, 129], [0, 130, 99, 126]),
                                              (8, 1, 64, [300], [5]), (4, 4, 128, [257, 385], [0, 128])])
def test_what_lies_behind_the_last_token(hq, hkv, d, new, ctx, flags):
    """NaN and infinities in the slots behind a sequence's tokens, in all other pages, and in page 0, which unused entries name."""
    c = Paged(new, ctx, hkv, d, seed=1)
    q = _q(int(c.q_start[-1]), hq, d, c.g)
    want, wl, st = _run(c, q, flags)
    assert st == 0
    used = torch.cat([c.slots(b, 0, c.ctx[b] + c.new[b]) for b in range(len(new))])
    free = torch.ones(c.num_pages * PAGE, dtype=torch.bool, device="cuda")
    free[used] = False
    for bad in (math.nan, math.inf, -math.inf):
        k, v = c.k.clone(), c.v.clone()
        k.view(-1, hkv, d)[free] = bad
        v.view(-1, hkv, d)[free] = bad
        out, lse, st = _run(c, q, flags, k=k, v=v)
        assert st == 0 and torch.equal(out, want) and torch.equal(lse, wl), bad


@pytest.mark.parametrize("flags", [0, 2])
def test_rows_and_sequences_left_alone(flags):
    from paper_2511_21699_b200 import _lib
    new, ctx = [3, 40, 1, 7], [10, 0, 33, 4]
    c = Paged(new, ctx, 2, 64)
    n = int(c.q_start[-1])
    lead, trail = 2, 6
    q = _q(lead + n + trail, 4, 64, c.g)
    cb = context(batch=4, n_q_heads=4, n_kv_heads=2, head_dim=64, flags=flags)
    base = Paged(new, ctx, 2, 64)

    def run(start=None, ctx_len=None, **kw):
        out, lse = torch.full_like(q, 7.0), torch.full((len(q), 4), 7.0, device="cuda")
        cb.cb_chunk_attn(q, c.k, c.v, c.block_table, cuda(c.q_start + lead if start is None else start), c.d_ctx if ctx_len is None else cuda(ctx_len), out=out,
                         lse=lse, **kw)
        return out, lse, cb.cb_poll_status()[0]

    def untouched(out, lse, rows):
        assert bool((out[rows] == 7).all()) and bool((lse[rows] == 7).all())
        keep = [r for r in range(lead, lead + n) if r not in rows]
        assert not bool((lse[keep] == 7).any())

    want, wl, st = run()
    assert st == 0
    untouched(want, wl, [0, 1] + list(range(lead + n, len(q))))
    _compare(want[lead:lead + n], wl[lead:lead + n], q[lead:lead + n], base, 64 ** -0.5)
    a = [lead + int(x) for x in c.q_start]
    out, lse, st = run(ctx_len=[10, 0, -1, 4])
    assert st == _lib.CB_ERR_INVALID_ARG
    untouched(out, lse, list(range(a[2], a[3])))
    out, lse, st = run(ctx_len=[10, 10 ** 6, 33, 2 ** 31 - 1])
    assert st == _lib.CB_ERR_KV_FULL
    untouched(out, lse, list(range(a[1], a[2])) + list(range(a[3], a[4])))
    out, lse, st = run(max_chunk=39)
    assert st == _lib.CB_ERR_INVALID_ARG
    untouched(out, lse, list(range(a[1], a[2])))
    out, lse, st = run(max_ctx=20, max_chunk=40)
    assert st == _lib.CB_ERR_KV_FULL
    untouched(out, lse, list(range(a[1], a[3])))
    assert torch.equal(out[a[0]:a[1]], want[a[0]:a[1]])
    big = len(q) + 5
    out, lse, st = run(start=[2, 5, 45, 46, big])                 # behind the last row
    assert st == _lib.CB_ERR_INVALID_ARG
    untouched(out, lse, list(range(a[3], a[4])))
    out, lse, st = run(start=[2, 5, 5, 5, 5])
    assert st == 0 and (out[5:] == 7).all() and torch.equal(out[2:5], want[2:5])
    # every sequence empty
    out, lse, st = run(start=[0, 0, 0, 0, 0])
    assert st == 0 and (out == 7).all() and (lse == 7).all()


@pytest.mark.parametrize("flags", [0, 2])
def test_pages_outside_the_pool_read_as_zeros(flags):
    c = Paged([5, 40], [100, 20], 2, 64)
    q = _q(45, 4, 64, c.g)
    bt = c.block_table.clone()
    for b, j, bad in ((0, 2, -1), (0, 4, c.num_pages), (1, 0, 2 ** 31 - 1), (1, 2, -2 ** 31)):
        c.k.view(-1, 2, 64)[c.slots(b, j * PAGE, j * PAGE + PAGE)] = 0
        c.v.view(-1, 2, 64)[c.slots(b, j * PAGE, j * PAGE + PAGE)] = 0
        bt[b, j] = bad
    want, wl, _ = _run(c, q, flags)
    c.block_table = bt
    out, lse, st = _run(c, q, flags)
    assert st == 0 and torch.equal(out, want) and torch.equal(lse, wl)


def test_pages_far_into_a_large_pool():
    """Elements past 2^31, and byte offsets past 2^32, in a pool of 2^18 + 64 pages of 16 x 8 x 64 (4.3 GB for keys and values each)."""
    pages, hkv, d = (1 << 18) + 64, 8, 64
    c = Paged([2, 30], [50, 200], hkv, d)
    k, v = (torch.zeros(pages, PAGE, hkv, d, device="cuda", dtype=BF) for _ in range(2))
    k[-c.num_pages:], v[-c.num_pages:] = c.k, c.v
    q = _q(32, 16, d, c.g)
    want, wl, _ = _run(c, q)
    c.block_table = c.block_table + (pages - c.num_pages)
    for flags in (0, 2):
        out, lse, st = _run(c, q, flags, k=k, v=v)
        assert st == 0
        if flags == 0:
            assert torch.equal(out, want) and torch.equal(lse, wl)
        else:
            _compare(out, lse, q, c, d ** -0.5)
    # and appending there
    cb = context(batch=2, n_q_heads=16, n_kv_heads=hkv, head_dim=d)
    kk, vv = (torch.randn(32, hkv, d, generator=c.g, device="cuda", dtype=BF) for _ in range(2))
    cb.cb_chunk_append(q, kk, vv, c.d_start, c.d_ctx, k, v, c.block_table)
    assert cb.cb_poll_status()[0] == 0
    tail_k, tail_v = k[-c.num_pages:].view(-1, hkv, d), v[-c.num_pages:].view(-1, hkv, d)
    at = torch.cat([c.slots(b, c.ctx[b], c.ctx[b] + c.new[b]) for b in range(2)])
    assert torch.equal(tail_k[at], kk) and torch.equal(tail_v[at], vv)


def test_equal_calls_give_equal_bits_and_share_a_context_with_tree_attention():
    """The same workspace serves both attentions in turn."""
    import workloads as W
    from tests.harness import Problem, device_attn_inputs, synthetic_trees
    cfg = W.CbConfig("both", 6, 2, 2, 64, 2, 40, 6, 0, 8, 2, 128, (200, 900), 100, 1.1, 0.3, (4, 8), 64)
    prob = Problem(cfg)
    d = device_attn_inputs(cfg, prob)
    _, _, mask, n = synthetic_trees(cfg, full=False)
    c = Paged([1, 90, 0, 300, 17, 1], [800, 90, 3, 0, 77, 3000], 2, 128)
    q = _q(int(c.q_start[-1]), 8, 128, c.g)
    cb = context(batch=6, max_nodes=40, n_q_heads=8, n_kv_heads=2, head_dim=128)
    tree = lambda: cb.cb_tree_attn(d["q"], d["k_pool"], d["v_pool"], d["block_table"], d["ctx_len"], d["k_tree"], d["v_tree"], cuda(mask.view(np.int32)), cuda(n),
                                   max_ctx=int(prob.ctx.max()))
    first, (want, wl, st) = tree(), _run(c, q, cb=cb)
    assert st == 0
    _compare(want, wl, q, c, 128 ** -0.5)
    for _ in range(5):
        out, lse, st = _run(c, q, cb=cb)
        assert st == 0 and torch.equal(out, want) and torch.equal(lse, wl)
        assert torch.equal(tree(), first)


def test_captured_and_on_another_stream():
    """A graph captured with one set of lengths and replayed with others within the bounds."""
    c = Paged([1, 20, 5], [300, 10, 700], 4, 64, spare_pages=10)
    q = _q(60, 8, 64, c.g)
    cb = context(batch=3, n_q_heads=8, n_kv_heads=4, head_dim=64)
    out, lse = torch.empty_like(q), torch.empty(60, 8, device="cuda")
    call = lambda **kw: cb.cb_chunk_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, out=out, lse=lse, max_chunk=32, max_ctx=900, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(stream=side)
    side.synchronize()
    _compare(out[:26], lse[:26], q[:26], c, 0.125)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    c.new, c.ctx = np.array([32, 0, 28]), np.array([200, 10, 641])
    c.q_start = np.concatenate([[0], np.cumsum(c.new)])
    c.d_start.copy_(cuda(c.q_start))
    c.d_ctx.copy_(cuda(c.ctx))
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert cb.cb_poll_status()[0] == 0
    _compare(out, lse, q, c, 0.125)


@pytest.mark.parametrize("hq,hkv,d,flags", [(8, 2, 64, 0), (8, 8, 128, 0), (8, 2, 128, 2)])
def test_prompt_in_chunks_then_tokens_then_a_tree(hq, hkv, d, flags):
    """The operators as a program runs them: prompts go in chunk by chunk, then single tokens, then a chain as a draft tree's only branch; each
    step against attention over the whole sequence computed from the projections."""
    B, total = 3, [150, 83, 40]
    rng = np.random.default_rng(1)
    g = torch.Generator(device="cuda").manual_seed(5)
    T = 12
    proj = [(torch.randn(t + T, hq + 2 * hkv, d, generator=g, device="cuda") * 1.2).to(BF) for t in total]
    wq, wk = ((1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(BF) for _ in range(2))
    table = rope_table(200, d)
    c = Paged([0] * B, [t + T for t in total], hkv, d)
    c.k.fill_(0)
    c.v.fill_(0)
    cb = context(batch=B, max_nodes=T, max_depth=T, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, flags=flags)
    kw = dict(rope=table, q_norm=wq, k_norm=wk)

    def prepared(got, x, w, pos):                                 # normed and rotated as the formula says
        z, bound = normed_and_turned(x, w, 1e-6, table, torch.as_tensor(pos, device="cuda"), False)
        assert bool(((got.to(F8) - z).abs() <= bound).all())

    def near(out, q, k, v, lo):                                   # attention of what was prepared
        want, _, bound, _ = attention(q, k, v, lo, d ** -0.5)
        assert bool(((out.to(F8) - want).abs() <= bound).all()), lo

    pool = lambda x, b, n: x.view(-1, hkv, d)[c.slots(b, 0, n)]
    ctx = np.zeros(B, np.int64)
    steps = 0
    while (ctx < total).any():
        left = np.array(total) - ctx
        new = np.where(rng.random(B) < 0.3, np.minimum(left, 1), np.minimum(left, rng.integers(0, 60, B)))
        if new.sum() == 0:
            continue
        start = np.concatenate([[0], np.cumsum(new)])
        x = torch.cat([proj[b][ctx[b]:ctx[b] + new[b]] for b in range(B)])
        d_start, d_ctx = cuda(start), cuda(ctx)
        q = cb.cb_chunk_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], d_start, d_ctx, c.k, c.v, c.block_table, **kw)
        out = cb.cb_chunk_attn(q, c.k, c.v, c.block_table, d_start, d_ctx, max_chunk=int(new.max()))
        for b in range(B):
            if new[b]:
                rows, end = slice(start[b], start[b + 1]), ctx[b] + new[b]
                prepared(q[rows], proj[b][ctx[b]:end, :hq], wq, np.arange(ctx[b], end))
                near(out[rows], q[rows], pool(c.k, b, end), pool(c.v, b, end), int(ctx[b]))
        ctx += new
        steps += 1
    assert steps > 4
    # the next T tokens as a chain of nodes
    x = torch.cat([proj[b][total[b]:] for b in range(B)])
    chain = np.tril(np.ones((T, T), np.int64))
    mask = (chain * (1 << np.arange(T))).sum(1)
    tree = dict(depth=cuda(np.tile(np.arange(T), (B, 1))), n_nodes=cuda([T] * B))
    q, kt, vt = cb.cb_tree_rope(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], tree, cuda(ctx), **kw)
    out = cb.cb_tree_attn(q, c.k, c.v, c.block_table, cuda(ctx), kt, vt, cuda(np.tile(mask[None, :, None], (B, 1, 1))), tree["n_nodes"])
    for b in range(B):
        prepared(pool(c.k, b, total[b]), proj[b][:total[b], hq:hq + hkv], wk, np.arange(total[b]))
        assert torch.equal(pool(c.v, b, total[b]), proj[b][:total[b], hq + hkv:])
        prepared(q[b], proj[b][total[b]:, :hq], wq, total[b] + np.arange(T))
        prepared(kt[b], proj[b][total[b]:, hq:hq + hkv], wk, total[b] + np.arange(T))
        near(out[b], q[b], torch.cat([pool(c.k, b, total[b]), kt[b]]), torch.cat([pool(c.v, b, total[b]), vt[b]]), total[b])
    # committing the whole chain leaves what appending it would have left
    after, ka, va = cuda(ctx), c.k.clone(), c.v.clone()
    cb.cb_kv_commit(ka, va, c.block_table, after, kt, vt, cuda([T - 1] * B), cuda(np.tile(np.arange(1, T + 1) % T, (B, 1))))
    cb.cb_chunk_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], cuda(np.arange(B + 1) * T), cuda(ctx), c.k, c.v, c.block_table, **kw)
    assert torch.equal(ka, c.k) and torch.equal(va, c.v) and after.tolist() == [t + T for t in total]
    assert cb.cb_poll_status()[0] == 0


def test_refused():
    from paper_2511_21699_b200 import CachebackError
    c = Paged([2, 1], [0, 3], 2, 64)
    q = _q(3, 4, 64, c.g)
    cb = context(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64)
    good = dict(q=q, k_pool=c.k, v_pool=c.v, block_table=c.block_table, q_start=c.d_start, ctx_len=c.d_ctx)
    for change, text in ((dict(q=q.float()), "q: expected dtype torch.bfloat16"), (dict(q=q[:, :2]), "q must be"), (dict(q=q.transpose(0, 1)), "q must be|contiguous"),
                         (dict(k_pool=c.k.cpu()), "CUDA"), (dict(v_pool=c.v[:1]), "v_pool must be"), (dict(block_table=c.block_table[:1]), "block_table"),
                         (dict(q_start=c.d_ctx), "q_start must be"), (dict(ctx_len=c.d_start), "ctx_len must be"), (dict(out=q), "invalid argument"),
                         (dict(out=q[:2]), "out must be"), (dict(lse=torch.empty(4, 3, device="cuda")), "lse must be"), (dict(max_chunk=-1), "invalid argument"),
                         (dict(max_ctx=-1), "invalid argument"), (dict(max_ctx=2 ** 31), "32-bit"),
                         (dict(q=torch.empty(3 * 4 * 64 + 1, device="cuda", dtype=BF)[1:].view(3, 4, 64)), "invalid argument")):
        with pytest.raises(CachebackError, match=text):
            cb.cb_chunk_attn(**{**good, **change})
    assert cb.cb_chunk_attn(**{**good, "q": q[:0], "q_start": cuda([0, 0, 0])}).shape == (0, 4, 64)
    assert cb.cb_poll_status()[0] == 0
