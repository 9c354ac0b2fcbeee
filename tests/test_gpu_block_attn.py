"""cb_block_attn and cb_block_tree_attn against softmax attention over the listed blocks in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests.block_refs import mask_words, masked_attention, positions, random_lists, random_trees
from tests.operator_refs import F8, PAGE, Paged, context, cuda

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
OK, INVALID, FULL = 0, 1, 8


def _q(shape, g, scale=1.5):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(BF)


def _run(c, q, lists, block, flags=0, hints=True, cb=None, scale=0.0):
    hkv, d = c.k.shape[2:]
    n, hq = q.shape[:2]
    cb = cb or context(batch=len(c.new), n_q_heads=hq, n_kv_heads=hkv, head_dim=d, flags=flags)
    out, lse = torch.full_like(q, 7.0), torch.full((n, hq), 7.0, device="cuda")
    cb.cb_block_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, cuda(lists), block=block, out=out, lse=lse, max_chunk=int(c.new.max()) if hints else 0,
                     max_ctx=int((c.new + c.ctx).max()) if hints else 0, scale=scale)
    return out, lse, cb.cb_poll_status()[0]


def _compare(out, lse, q, c, lists, block, scale, seqs=None):
    hkv, d = c.k.shape[2:]
    G = q.shape[1] // hkv
    k, v = c.k.view(-1, hkv, d), c.v.view(-1, hkv, d)
    for b in range(len(c.new)) if seqs is None else seqs:
        lo, hi, n = c.q_start[b], c.q_start[b + 1], int(c.new[b])
        if n == 0:
            continue
        for h in range(hkv):
            seen = positions(lists[b, h][lists[b, h] >= 0], int(c.ctx[b]), block)
            pos = np.concatenate([seen, c.ctx[b] + np.arange(n)])
            at = cuda(c.bt[b, pos // PAGE] * PAGE + pos % PAGE, torch.int64)
            vis = cuda(pos[None] <= (c.ctx[b] + np.arange(n))[:, None], torch.bool)
            ref, rl, b_out, b_lse = masked_attention(q[lo:hi, h * G:h * G + G], k[at, h], v[at, h], vis, scale)
            off, loff = (out[lo:hi, h * G:h * G + G].to(F8) - ref).abs(), (lse[lo:hi, h * G:h * G + G].to(F8) - rl).abs()
            assert bool((off <= b_out).all()), (b, h, n, int(c.ctx[b]), float((off - b_out).max()), float(off.max()))
            assert bool((loff <= b_lse).all()), (b, h, float((loff - b_lse).max()), float(loff.max()))


SHAPES = [
    # hq, hkv, d, block, n_select, new, ctx
    (8, 8, 64, 64, 4, [1], [0]),
    (8, 8, 64, 16, 3, [1], [1000]),
    (32, 8, 128, 64, 32, [1] * 9, [0, 1, 63, 64, 65, 2048, 2049, 2112, 9000]),
    (32, 32, 128, 64, 5, [1], [4096]),
    (64, 8, 128, 128, 6, [1, 0, 1], [3000, 77, 5000]),
    (28, 4, 128, 32, 9, [3, 18, 19, 36, 37], [0, 5, 2500, 1, 1280]),
    (5, 1, 64, 16, 20, [25, 26, 51, 1], [0, 1000, 300, 3000]),
    (48, 3, 64, 64, 3, [8, 9, 40], [7, 0, 3000]),
    (16, 1, 128, 64, 33, [1, 1, 2], [30000, 2113, 2111]),
    (8, 8, 128, 32, 4, [128, 127, 129, 256, 257, 1], [0, 0, 1, 300, 1280, 129]),
    (16, 4, 64, 16, 50, [309, 0, 1, 64, 200, 33], [3, 9, 1203, 640, 0, 3100]),
    (6, 2, 64, 128, 2, [700, 1], [1513, 0]),
    (40, 40, 64, 32, 7, [15, 16, 17], [1, 900, 15]),
    (3, 3, 128, 16, 1, [1, 2], [500, 15]),
]


@pytest.mark.parametrize("hq,hkv,d,block,K,new,ctx", SHAPES)
@pytest.mark.parametrize("flags", [0, 2])
def test_shapes(hq, hkv, d, block, K, new, ctx, flags):
    c = Paged(new, ctx, hkv, d, seed=hq + len(new))
    q = _q((int(c.q_start[-1]), hq, d), c.g)
    lists = random_lists(c.ctx, hkv, K, block, seed=K)
    for hints in (True, False):
        out, lse, st = _run(c, q, lists, block, flags, hints)
        assert st == OK
        _compare(out, lse, q, c, lists, block, d ** -0.5)


def test_many_sequences():
    rng = np.random.default_rng(2)
    new = np.where(rng.random(300) < 0.8, 1, rng.integers(0, 70, 300))
    c = Paged(new, rng.integers(0, 2000, 300), 2, 64)
    q = _q((int(c.q_start[-1]), 8, 64), c.g)
    lists = random_lists(c.ctx, 2, 6, 64, seed=1)
    out, lse, st = _run(c, q, lists, 64)
    assert st == OK
    _compare(out, lse, q, c, lists, 64, 64 ** -0.5)
    for b in range(300):                                                     # rows of no sequence: none here, and none was left out
        assert not bool((out[c.q_start[b]:c.q_start[b + 1]] == 7.0).all(-1).any())


def _tree_case(hq, hkv, d, T, n, ctx, seed=0, vis=None):
    ctx, n = np.asarray(ctx), np.asarray(n)
    c = Paged(0 * ctx, ctx, hkv, d, seed=seed)
    B = len(ctx)
    # what lies in the last page's free slots is finite, as tree attention wants it
    q, kt, vt = _q((B, T, hq, d), c.g), _q((B, T, hkv, d), c.g, 1.0), _q((B, T, hkv, d), c.g, 1.0)
    v, words = random_trees(B, T, n, seed) if vis is None else (vis, mask_words(vis))
    return c, q, kt, vt, v, words, cuda(n)


def _run_tree(c, q, kt, vt, words, n, lists, block, flags=0, hints=True, cb=None, scale=0.0):
    B, T, hq, d = q.shape
    cb = cb or context(batch=B, n_q_heads=hq, n_kv_heads=kt.shape[2], head_dim=d, max_nodes=T, flags=flags)
    out, lse = torch.full_like(q, 7.0), torch.full((B, hq, T), 7.0, device="cuda")
    cb.cb_block_tree_attn(q, c.k, c.v, c.block_table, c.d_ctx, kt, vt, words, n, cuda(lists), block=block, out=out, lse=lse,
                          max_ctx=int(c.ctx.max()) if hints else 0, scale=scale)
    return out, lse, cb.cb_poll_status()[0]


def _compare_tree(out, lse, q, c, kt, vt, vis, n, lists, block, scale):
    B, T, hq, d = q.shape
    hkv = kt.shape[2]
    G = hq // hkv
    k, v = c.k.view(-1, hkv, d), c.v.view(-1, hkv, d)
    for b in range(B):
        m = int(n[b])
        assert bool((out[b, m:] == 0).all()) and bool((lse[b, :, m:] == 0).all())
        if m == 0:
            continue
        for h in range(hkv):
            pos = positions(lists[b, h][lists[b, h] >= 0], int(c.ctx[b]), block)
            at = cuda(c.bt[b, pos // PAGE] * PAGE + pos % PAGE, torch.int64)
            seen = np.concatenate([np.ones((m, len(pos)), bool), vis[b, :m, :m]], 1)
            ref, rl, b_out, b_lse = masked_attention(q[b, :m, h * G:h * G + G], torch.cat((k[at, h], kt[b, :m, h])), torch.cat((v[at, h], vt[b, :m, h])),
                                                     cuda(seen, torch.bool), scale)
            off, loff = (out[b, :m, h * G:h * G + G].to(F8) - ref).abs(), (lse[b, h * G:h * G + G, :m].t().to(F8) - rl).abs()
            assert bool((off <= b_out).all()), (b, h, m, int(c.ctx[b]), float((off - b_out).max()), float(off.max()))
            assert bool((loff <= b_lse).all()), (b, h, float((loff - b_lse).max()), float(loff.max()))


@pytest.mark.parametrize("hq,hkv,d,block,K,T,n,ctx", [
    (8, 8, 64, 64, 4, 1, [1, 1, 0], [0, 1000, 5]),
    (32, 8, 128, 64, 32, 64, [64, 64, 33, 1], [9000, 2048, 2049, 0]),
    (64, 8, 128, 128, 3, 128, [128, 127, 90], [3000, 384, 385]),
    (16, 4, 64, 16, 9, 61, [61, 0, 13, 60], [1, 800, 5003, 143]),
    (28, 4, 128, 32, 20, 37, [37, 18, 19], [1000, 640, 641]),
    (16, 1, 128, 64, 10, 128, [128, 1, 65], [700, 20000, 640]),
    (5, 1, 64, 32, 6, 31, [31, 25, 26, 1], [5, 192, 193, 2000]),
    (40, 40, 64, 64, 2, 96, [96, 95], [129, 1280]),
])
@pytest.mark.parametrize("flags", [0, 2])
def test_trees(hq, hkv, d, block, K, T, n, ctx, flags):
    c, q, kt, vt, vis, words, dn = _tree_case(hq, hkv, d, T, n, ctx, seed=T)
    lists = random_lists(c.ctx, hkv, K, block, seed=K)
    for hints in (True, False):
        out, lse, st = _run_tree(c, q, kt, vt, words, dn, lists, block, flags, hints)
        assert st == OK
        _compare_tree(out, lse, q, c, kt, vt, vis, n, lists, block, d ** -0.5)


def test_all_blocks_listed_is_dense_attention():
    """With room for every block the lists say nothing: the rows are those of the dense calls, within both calls' bounds."""
    c, q, kt, vt, vis, words, dn = _tree_case(16, 4, 128, 40, [40, 7, 25], [700, 0, 129])
    lists = random_lists(c.ctx, 4, 16, 64, seed=0)
    out, lse, _ = _run_tree(c, q, kt, vt, words, dn, lists, 64)
    cb = context(batch=3, n_q_heads=16, n_kv_heads=4, head_dim=128, max_nodes=40)
    dl = torch.empty_like(lse)
    dense = cb.cb_tree_attn(q, c.k, c.v, c.block_table, c.d_ctx, kt, vt, words, dn, lse=dl)
    assert float((out.float() - dense.float()).abs().max()) <= 2.0 ** -6 and float((lse - dl).abs().max()) <= 1e-4
    c = Paged([40, 1, 90], [700, 300, 0], 4, 128)
    q = _q((131, 16, 128), c.g)
    lists = random_lists(c.ctx, 4, 16, 64, seed=0)
    out, lse, _ = _run(c, q, lists, 64)
    cb = context(batch=3, n_q_heads=16, n_kv_heads=4, head_dim=128)
    dl = torch.empty_like(lse)
    dense = cb.cb_chunk_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, lse=dl)
    assert float((out.float() - dense.float()).abs().max()) <= 2.0 ** -6 and float((lse - dl).abs().max()) <= 1e-4


@pytest.mark.parametrize("flags", [0, 2])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 3, 130]])
def test_what_lies_behind_the_last_token_does_not_matter(new, flags):
    """NaN and infinities in the slots of the last page behind a sequence's tokens, and in all pages that no list names."""
    c = Paged(new, [1003, 65, 700], 2, 64)
    q = _q((int(c.q_start[-1]), 8, 64), c.g)
    lists = random_lists(c.ctx, 2, 5, 64, seed=3)
    lists[:, 1] = lists[:, 0]                                                # a page serves both heads
    keep = torch.zeros(c.num_pages * PAGE, dtype=torch.bool, device="cuda")
    for b in range(3):
        pos = np.concatenate([positions(lists[b, 0][lists[b, 0] >= 0], int(c.ctx[b]), 64), c.ctx[b] + np.arange(new[b])])
        keep[cuda(c.bt[b, pos // PAGE] * PAGE + pos % PAGE, torch.int64)] = True
    k0, v0 = c.k.clone(), c.v.clone()
    for bad in (math.nan, math.inf, -math.inf):
        c.k.copy_(torch.where(keep.view(-1, PAGE, 1, 1), k0, bad))
        c.v.copy_(torch.where(keep.view(-1, PAGE, 1, 1), v0, bad))
        out, lse, st = _run(c, q, lists, 64, flags)
        assert st == OK
        _compare(out, lse, q, c, lists, 64, 64 ** -0.5)


@pytest.mark.parametrize("flags", [0, 2])
def test_scores_far_apart_and_rising(flags):
    """Each block's scores above the one before by far more than fp32's exponent, for the last ones; and a far score in the first."""
    for new in ([1], [33]):
        for sign in (1, -1):
            c = Paged(new, [2000], 1, 128)
            c.k.mul_(0.05)
            line = torch.linspace(0, 40 * sign, 2100, device="cuda")
            flat = c.k.view(-1, 1, 128)
            at = c.slots(0, 0, 2000 + new[0])
            flat[at, :, 0] = line[:len(at), None].to(BF)
            q = _q((new[0], 4, 128), c.g, 0.1)
            q[..., 0] = 100.0
            lists = random_lists(c.ctx, 1, 10, 64, seed=5)
            out, lse, st = _run(c, q, lists, 64, flags)
            assert st == OK
            _compare(out, lse, q, c, lists, 64, 128 ** -0.5)


@pytest.mark.parametrize("flags", [0, 2])
def test_rows_of_no_sequence_are_left_and_bad_sequences_too(flags):
    c = Paged([2, 3, 1, 40], [500, 600, 700, 800], 2, 64)
    n = int(c.q_start[-1]) + 9
    q = _q((n, 4, 64), c.g)
    lists = random_lists(c.ctx, 2, 4, 64, seed=1)
    out, lse, st = _run(c, q, lists, 64, flags)
    assert st == OK and bool((out[n - 9:] == 7).all()) and bool((lse[n - 9:] == 7).all())
    _compare(out, lse, q, c, lists, 64, 0.125)
    keep = c.d_ctx.clone()
    for bad, why in ((-1, INVALID), (16 * c.bt.shape[1], FULL), ((1 << 31) - 1, FULL), (-(1 << 31), INVALID)):
        c.d_ctx.copy_(keep)
        c.d_ctx[1] = bad
        for hints in (True, False):
            out, lse, st = _run(c, q, lists, 64, flags, hints)
            assert st == why and bool((out[2:5] == 7).all()) and bool((lse[2:5] == 7).all())
            _compare(out, lse, q, c, lists, 64, 0.125, seqs=(0, 2, 3))
    c.d_ctx.copy_(keep)
    c.d_start.copy_(cuda([0, 2, 1, 6, 46]))
    out, lse, st = _run(c, q, lists, 64, flags, False)
    assert st == INVALID
    _compare(out, lse, q, c, lists, 64, 0.125, seqs=(3,))                    # (row 1 lies in the ranges of sequences 0 and 2)


@pytest.mark.parametrize("flags", [0, 2])
@pytest.mark.parametrize("new", [1, 30])
def test_pages_and_blocks_that_do_not_exist_read_as_zeros(new, flags):
    c = Paged([new], [1000], 2, 64)
    q = _q((new, 4, 64), c.g)
    lists = random_lists(c.ctx, 2, 6, 64, seed=1)
    lists[0, 0, 0], lists[0, 1, 0] = 3, 3
    c.v.fill_(1.0)
    ref_k, ref_v = c.k.clone(), c.v.clone()
    at = c.slots(0, 192, 208)
    c.k.view(-1, 2, 64)[at], c.v.view(-1, 2, 64)[at] = 0, 0
    for bad in (-1, c.num_pages, 1 << 30):
        page = int(c.block_table[0, 12])
        want = _run(c, q, lists, 64, flags)
        c.block_table[0, 12] = bad
        c.k, ref_k = ref_k, c.k
        c.v, ref_v = ref_v, c.v
        got = _run(c, q, lists, 64, flags)
        c.k, ref_k = ref_k, c.k
        c.v, ref_v = ref_v, c.v
        c.block_table[0, 12] = page
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    c.k.zero_()
    c.v.zero_()
    want = _run(c, q, lists, 64, flags)
    for bad in (-1, 16, 1 << 30, -(1 << 31), (1 << 31) - 1):                # block 15 is the newest one
        lists[0, :, 1] = bad
        got = _run(c, q, lists, 64, flags)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("flags", [0, 2])
def test_tree_rows_whose_mask_leaves_only_the_context_or_nothing(flags):
    vis = np.zeros((3, 20, 20), bool)
    vis[0, np.arange(0, 20, 2), 0] = True
    c, q, kt, vt, vis, words, n = _tree_case(8, 2, 64, 20, [20, 20, 20], [300, 0, 129], vis=vis)
    lists = random_lists(c.ctx, 2, 3, 64, seed=0)
    out, lse, st = _run_tree(c, q, kt, vt, words, n, lists, 64, flags)
    assert st == OK
    _compare_tree(out, lse, q, c, kt, vt, vis, [20, 20, 20], lists, 64, 0.125)


@pytest.mark.parametrize("scale", [1.0, 0.01])
def test_scale(scale):
    c = Paged([1, 20], [900, 100], 2, 64)
    q = _q((21, 4, 64), c.g, 0.5)
    lists = random_lists(c.ctx, 2, 5, 32, seed=0)
    out, lse, st = _run(c, q, lists, 32, scale=scale)
    _compare(out, lse, q, c, lists, 32, scale)


@pytest.mark.parametrize("new", [[1] * 7, [50, 1, 200]])
def test_equal_calls_give_equal_bits(new):
    rng = np.random.default_rng(4)
    c = Paged(new, rng.integers(0, 9000, len(new)), 8, 128)
    q = _q((int(c.q_start[-1]), 32, 128), c.g)
    lists = random_lists(c.ctx, 8, 32, 64, seed=0)
    cb = context(batch=len(new), n_q_heads=32, n_kv_heads=8, head_dim=128)
    first = _run(c, q, lists, 64, cb=cb)
    for _ in range(10):
        again = _run(c, q, lists, 64, cb=cb)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
