"""cb_chunk_append and cb_tree_rope against the formula in 64 bits: norm, rotation, where rows go and what stays as it was."""
import numpy as np
import pytest
import torch

from tests.operator_refs import BF16_HALF, F8, PAGE, Paged, context, cuda, normed_and_turned, rope_table

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _rows(n, heads, d, g, scale=1.5):
    return torch.randn(n, heads, d, generator=g, device="cuda", dtype=BF) * scale


def _norms(d, g, on):
    return tuple((1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(BF) for _ in range(2)) if on else (None, None)


def _check(got, x, w, eps, table, pos, inter, what):
    ref, bound = normed_and_turned(x, w, eps, table, pos, inter)
    off = (got.to(F8) - ref).abs()
    assert bool((off <= bound).all()), (what, float((off - bound).max()))


@pytest.mark.parametrize("hq,hkv,d,rot,norm,inter,new,ctx", [
    (32, 8, 128, 128, True, False, [1, 1, 1, 1], [0, 15, 16, 4001]),
    (8, 8, 64, 64, True, True, [0, 17, 0, 1, 33], [0, 0, 5, 31, 15]),
    (40, 40, 128, 64, False, False, [5], [1]),
    (28, 4, 64, 32, False, True, [300, 0, 1], [0, 0, 0]),
    (5, 1, 128, 16, True, False, [2, 3], [14, 15]),
    (16, 4, 64, 48, True, True, [16, 16, 16], [0, 16, 8]),
    (3, 3, 64, 0, True, False, [4, 1], [9, 0]),
    (7, 7, 128, 0, False, False, [6], [3]),
    (64, 8, 128, 128, True, False, [700, 1, 800], [5, 100, 0]),   # two groups of heads a warp, not all of them there
    (64, 8, 128, 64, True, True, [2100], [3]),                    # four
    (21, 7, 64, 64, True, False, [9000], [0]),
    (40, 40, 64, 32, False, False, [3000], [1000]),
])
@pytest.mark.parametrize("packed", [True, False])
def test_append(hq, hkv, d, rot, norm, inter, new, ctx, packed):
    c = Paged(new, ctx, hkv, d, seed=hq + d)
    n = int(c.q_start[-1])
    qkv = _rows(n, hq + 2 * hkv, d, c.g)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    table = rope_table(max(4200, max(new) + max(ctx)), rot) if rot else None
    wq, wk = _norms(d, c.g, norm)
    cb = context(batch=len(new), n_q_heads=hq, n_kv_heads=hkv, head_dim=d)
    kp, vp = c.k.clone(), c.v.clone()
    out = cb.cb_chunk_append(q, k, v, c.d_start, c.d_ctx, kp, vp, c.block_table, rope=table, q_norm=wq, k_norm=wk, eps=1e-5, interleaved=inter)
    assert cb.cb_poll_status()[0] == 0
    pos = cuda(np.concatenate([np.arange(a, a + m) for a, m in zip(ctx, new)]), torch.int64)
    _check(out, q, wq, 1e-5, table, pos, inter, "q")
    at = torch.cat([c.slots(b, ctx[b], ctx[b] + new[b]) for b in range(len(new))])
    _check(kp.view(-1, hkv, d)[at], k, wk, 1e-5, table, pos, inter, "k")
    assert torch.equal(vp.view(-1, hkv, d)[at], v)
    rest = torch.ones(kp.shape[0] * PAGE, dtype=torch.bool, device="cuda")
    rest[at] = False
    for got, was in ((kp, c.k), (vp, c.v)):                       # every other slot as it was
        assert torch.equal(got.view(-1, hkv, d)[rest], was.view(-1, hkv, d)[rest])


def test_append_in_place_many_sequences_and_rows_of_no_sequence():
    """2,100 sequences (three rounds of the search), rows before the first and behind the last left alone, queries in place."""
    rng = np.random.default_rng(3)
    new = rng.integers(0, 4, 2100)
    new[:40] = 0
    ctx = rng.integers(0, 40, 2100)
    c = Paged(new, ctx, 2, 64)
    lead, trail = 5, 9
    n = int(c.q_start[-1])
    q, k, v = (_rows(lead + n + trail, h, 64, c.g) for h in (4, 2, 2))
    was, kp, vp = q.clone(), c.k.clone(), c.v.clone()
    table = rope_table(64, 64)
    cb = context(batch=2100, n_q_heads=4, n_kv_heads=2, head_dim=64)
    got = cb.cb_chunk_append(q, k, v, cuda(c.q_start + lead), c.d_ctx, kp, vp, c.block_table, rope=table, q_out=q)
    assert got is q and cb.cb_poll_status()[0] == 0
    pos = cuda(np.concatenate([np.arange(a, a + m) for a, m in zip(ctx, new)]), torch.int64)
    _check(q[lead:lead + n], was[lead:lead + n], None, 0, table, pos, False, "q")
    assert torch.equal(q[:lead], was[:lead]) and torch.equal(q[lead + n:], was[lead + n:])
    at = torch.cat([c.slots(b, ctx[b], ctx[b] + new[b]) for b in range(2100)])
    assert torch.equal(vp.view(-1, 2, 64)[at], v[lead:lead + n])
    rest = torch.ones(vp.shape[0] * PAGE, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(vp.view(-1, 2, 64)[rest], c.v.view(-1, 2, 64)[rest]) and torch.equal(kp.view(-1, 2, 64)[rest], c.k.view(-1, 2, 64)[rest])


def test_append_leaves_sequences_alone_that_do_not_fit():
    from paper_2511_21699_b200 import _lib
    new, ctx = [3, 2, 4, 2], [0, 31, 0, 5]
    c = Paged(new, ctx, 1, 64, width=2)                           # two pages: sequence 1 would need 33 tokens
    q, k, v = (_rows(11, h, 64, c.g) for h in (2, 1, 1))
    cb = context(batch=4, n_q_heads=2, n_kv_heads=1, head_dim=64)

    def run(expect, d_ctx=None, table=None, bt=None):
        kp, vp, out = c.k.clone(), c.v.clone(), torch.full((11, 2, 64), 7.0, device="cuda", dtype=BF)
        cb.cb_chunk_append(q, k, v, c.d_start, d_ctx if d_ctx is not None else c.d_ctx, kp, vp, c.block_table if bt is None else bt, rope=table, q_out=out)
        assert cb.cb_poll_status()[0] == expect
        changed = (vp != c.v).flatten(2).any(-1).view(-1)
        return out, changed

    out, changed = run(_lib.CB_ERR_KV_FULL)
    assert (out[3:5] == 7).all() and not (out[:3] == 7).all() and torch.equal(out[5:], q[5:])
    assert int(changed.sum()) == 9                                # 3 + 4 + 2 slots
    c.ctx[1] = 0
    ok = cuda([0, 0, 0, 5])
    out, changed = run(_lib.CB_ERR_INVALID_ARG, cuda([0, 0, -1, 5]))               # a negative length
    assert (out[5:9] == 7).all() and int(changed.sum()) == 3 + 2 + 2
    out, changed = run(_lib.CB_ERR_INVALID_ARG, ok, rope_table(6, 16))             # the last row's position is 6
    assert (out[10] == 7).all() and int(changed.sum()) == 10 and not (out[9] == 7).all()
    was = c.d_start
    for start, left in (([0, 3, 5, 9, 50], range(9, 11)), ([-3, 3, 5, 9, 11], range(3))):        # a range that is not of these rows
        c.d_start = cuda(start)
        out, changed = run(_lib.CB_ERR_INVALID_ARG, ok)
        assert (out[list(left)] == 7).all() and int(changed.sum()) == 11 - len(left)
    c.d_start = was
    bt = c.block_table.clone()
    bt[0, 0], bt[2, 0] = c.num_pages, -5
    out, changed = run(_lib.CB_ERR_INVALID_ARG, ok, None, bt)
    assert (out[:3] == 7).all() and (out[5:9] == 7).all() and int(changed.sum()) == 4


@pytest.mark.parametrize("hq,hkv,d,T,rot,norm,inter", [(32, 8, 128, 64, 128, True, False), (16, 4, 64, 61, 32, False, True), (8, 8, 64, 1, 64, True, True),
                                                       (5, 1, 128, 128, 96, True, False), (64, 8, 128, 128, 128, True, False), (200, 200, 128, 128, 128, True, True)])
def test_tree(hq, hkv, d, T, rot, norm, inter):
    B = 5
    g = torch.Generator(device="cuda").manual_seed(T)
    rng = np.random.default_rng(T)
    n = np.array([T, 1, 0, max(1, T // 2), max(1, T - 1)])
    dep = rng.integers(0, 9, (B, T))
    dep[np.arange(T)[None] >= n[:, None]] = -1
    ctx = np.array([0, 3000, 7, 16, 991])
    qkv = _rows(B * T, hq + 2 * hkv, d, g)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    table = rope_table(3009, rot)
    wq, wk = _norms(d, g, norm)
    cb = context(batch=B, max_nodes=T, n_q_heads=hq, n_kv_heads=hkv, head_dim=d)
    tree = dict(depth=cuda(dep), n_nodes=cuda(n))
    got = cb.cb_tree_rope(q, k, v, tree, cuda(ctx), rope=table, q_norm=wq, k_norm=wk, interleaved=inter)
    assert cb.cb_poll_status()[0] == 0
    live = cuda(np.arange(T)[None] < n[:, None], torch.bool).view(-1)
    pos = cuda((ctx[:, None] + dep).clip(0).reshape(-1), torch.int64)[live]
    for x, y, w in zip((q, k), got, (wq, wk)):
        y = y.view(B * T, -1, d)
        _check(y[live], x[live], w, 1e-6, table, pos, inter, "tree")
        assert (y[~live] == 0).all()
    y = got[2].view(B * T, -1, d)
    assert torch.equal(y[live], v[live]) and (y[~live] == 0).all()
    # in place, and a node behind the table's end
    k2 = k.contiguous()
    out = cb.cb_tree_rope(q, k2, v, tree, cuda(ctx), rope=table[:3000].contiguous(), q_norm=wq, k_norm=wk, interleaved=inter, k_out=k2.view(B, T, hkv, d))
    from paper_2511_21699_b200 import _lib
    assert cb.cb_poll_status()[0] == _lib.CB_ERR_INVALID_ARG
    assert torch.equal(out[1][0], got[1][0]) and torch.equal(out[1][3:], got[1][3:]) and (out[1][1] == 0).all() and (out[0][1] == 0).all()


def test_refused():
    from paper_2511_21699_b200 import CachebackError
    c = Paged([2, 1], [0, 3], 2, 64)
    q, k, v = (_rows(3, h, 64, c.g) for h in (4, 2, 2))
    cb = context(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64)
    good = dict(q=q, k=k, v=v, q_start=c.d_start, ctx_len=c.d_ctx, k_pool=c.k, v_pool=c.v, block_table=c.block_table, rope=rope_table(8, 64))
    kp = c.k.clone()
    for change, text in ((dict(q=q.float()), "q: expected dtype torch.bfloat16"), (dict(k=k[:2]), "k must be"), (dict(v=v.transpose(1, 2)), "v must be"),
                         (dict(q=q.cpu()), "CUDA"), (dict(q_start=c.d_start[:2]), "q_start must be"), (dict(ctx_len=c.d_ctx.long()), "dtype torch.int32"),
                         (dict(k_pool=c.k[:, :8]), "k_pool must be"), (dict(v_pool=c.v[1:]), "v_pool must be"), (dict(block_table=c.block_table[:1]), "block_table"),
                         (dict(rope=rope_table(8, 64).double()), "rope"), (dict(rope=rope_table(8, 24)), "invalid argument"),
                         (dict(rope=rope_table(8, 128)), "invalid argument"), (dict(q_norm=torch.ones(32, device="cuda", dtype=BF)), "q_norm must be"),
                         (dict(q_norm=torch.ones(64, device="cuda", dtype=BF), eps=-1.0), "invalid argument"),
                         (dict(q=torch.empty(3, 4, 68, device="cuda", dtype=BF)[..., 2:66]), "invalid argument|contiguous within"),
                         (dict(q_out=q[:, :2]), "q_out must be"), (dict(q=q[0]), "q must be")):
        with pytest.raises(CachebackError, match=text):
            cb.cb_chunk_append(**{**good, **change})
    assert torch.equal(c.k, kp)
    cb.cb_chunk_append(q[:0], k[:0], v[:0], cuda([0, 0, 0]), c.d_ctx, c.k, c.v, c.block_table)       # nothing to do
    assert torch.equal(c.k, kp) and cb.cb_poll_status()[0] == 0
    with pytest.raises(CachebackError, match="q must be"):
        cb.cb_tree_rope(q, k, v, dict(depth=cuda([[0], [0]]), n_nodes=cuda([1, 1])), c.d_ctx)       # three rows for two nodes
    cb.close()
    with pytest.raises(CachebackError, match="invalid argument"):
        cb.cb_chunk_append(**good)
