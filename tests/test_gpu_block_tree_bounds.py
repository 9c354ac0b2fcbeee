"""cb_block_tree_attn: sequences whose lengths are out of their bounds, pages and blocks that do not exist."""
import numpy as np
import pytest
import torch

from tests.block_refs import random_lists
from tests.operator_refs import cuda
from tests.test_gpu_block_attn import _compare_tree, _run_tree, _tree_case

pytestmark = pytest.mark.gpu
OK, INVALID, FULL = 0, 1, 8
HUGE, LEAST = (1 << 31) - 1, -(1 << 31)


# one row tile and CTAs that share a unit; several row tiles; more sequences than a warp has lanes
@pytest.mark.parametrize("hq,hkv,d,T,B", [(4, 2, 64, 20, 3), (32, 4, 128, 64, 4), (8, 4, 64, 61, 40), (2, 2, 128, 9, 70)])
@pytest.mark.parametrize("flags", [0, 2])
def test_lengths_out_of_their_bounds(hq, hkv, d, T, B, flags):
    rng = np.random.default_rng(B)
    ctx, n = rng.integers(0, 1500, B), rng.integers(1, T + 1, B)
    ctx[0] = 1500
    at = B - 2
    c, q, kt, vt, vis, words, dn = _tree_case(hq, hkv, d, T, n, ctx, seed=T)
    lists = random_lists(c.ctx, hkv, 5, 64, seed=0)
    room = 16 * c.bt.shape[1]
    for hints in (True, False):
        over = 1501 if hints else room + 1
        for what, bad, why in (("ctx", -1, INVALID), ("ctx", LEAST, INVALID), ("ctx", over, FULL), ("ctx", HUGE, FULL), ("n", -1, INVALID), ("n", T + 1, INVALID),
                               ("n", HUGE, INVALID), ("n", LEAST, INVALID), ("both", -1, INVALID), ("neither", 0, OK)):
            keep, dn2 = c.d_ctx.clone(), dn.clone()
            if what in ("ctx", "both"):
                c.d_ctx[at] = bad
            if what in ("n", "both"):
                dn2[at] = bad
            out, lse, st = _run_tree(c, q, kt, vt, words, dn2, lists, 64, flags, hints)
            c.d_ctx.copy_(keep)
            assert st == why, (what, bad, hints)
            m = n.copy()
            if what != "neither":
                m[at] = 0                                                    # its rows and log-sums are zero, as of a tree without nodes
            _compare_tree(out, lse, q, c, kt, vt, vis, m, lists, 64, d ** -0.5)
    keep = c.d_ctx.clone()                                                   # a tree without nodes has nothing to be wrong with
    for bad in (-1, HUGE):
        dn2, m = dn.clone(), n.copy()
        dn2[at], m[at] = 0, 0
        c.d_ctx[at] = bad
        out, lse, st = _run_tree(c, q, kt, vt, words, dn2, lists, 64, flags)
        assert st == OK
        c.d_ctx.copy_(keep)
        _compare_tree(out, lse, q, c, kt, vt, vis, m, lists, 64, d ** -0.5)


@pytest.mark.parametrize("flags", [0, 2])
def test_the_bound_is_of_the_cached_tokens_alone(flags):
    c, q, kt, vt, vis, words, dn = _tree_case(8, 2, 64, 30, [30, 30], [640, 17])
    lists = random_lists(c.ctx, 2, 4, 32, seed=0)
    out, lse, st = _run_tree(c, q, kt, vt, words, dn, lists, 32, flags)      # the bound is 640, cached and new are 670
    assert st == OK
    _compare_tree(out, lse, q, c, kt, vt, vis, [30, 30], lists, 32, 0.125)


@pytest.mark.parametrize("flags", [0, 2])
@pytest.mark.parametrize("hq,T", [(4, 12), (16, 50)])
def test_pages_and_blocks_that_do_not_exist_read_as_zeros(hq, T, flags):
    c, q, kt, vt, vis, words, dn = _tree_case(hq, 2, 64, T, [T], [1000])
    lists = random_lists(c.ctx, 2, 6, 64, seed=1)
    lists[0, :, 0] = 3
    k0, v0 = c.k.clone(), c.v.clone()
    at = c.slots(0, 192, 208)
    page = int(c.block_table[0, 12])
    c.k.view(-1, 2, 64)[at], c.v.view(-1, 2, 64)[at] = 0, 0
    want = _run_tree(c, q, kt, vt, words, dn, lists, 64, flags)
    _compare_tree(*want[:2], q, c, kt, vt, vis, [T], lists, 64, 0.125)
    c.k.copy_(k0)
    c.v.copy_(v0)
    for bad in (-1, c.num_pages, 1 << 30, LEAST):
        c.block_table[0, 12] = bad
        got = _run_tree(c, q, kt, vt, words, dn, lists, 64, flags)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    c.block_table[0, 12] = page
    at = c.slots(0, 192, 256)
    c.k.view(-1, 2, 64)[at], c.v.view(-1, 2, 64)[at] = 0, 0
    want = _run_tree(c, q, kt, vt, words, dn, lists, 64, flags)
    c.k.copy_(k0)
    c.v.copy_(v0)
    for bad in (-1, 16, 1 << 30, LEAST, HUGE):                               # block 15 is the newest one
        wrong = lists.copy()
        wrong[0, :, 0] = bad
        got = _run_tree(c, q, kt, vt, words, dn, wrong, 64, flags)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
