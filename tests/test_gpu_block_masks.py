"""cb_block_tree_attn: masks of any form, against softmax attention over the listed blocks and the nodes that a row's mask names, in 64 bits."""
import numpy as np
import pytest
import torch

from tests.block_refs import random_lists
from tests.test_gpu_block_attn import _compare_tree, _run_tree, _tree_case

pytestmark = pytest.mark.gpu
OK = 0


def _masks(kind, B, T):
    """Visible [B, T, T]: which of the first 32 nodes rows see decides where a running maximum starts."""
    rng = np.random.default_rng(T)
    vis = np.zeros((B, T, T), bool)
    for i in range(T):
        if kind == "itself":                                                 # rows 32 .. name no node below 32
            vis[:, i, i] = True
        elif kind == "the last":                                             # no row names any but one node
            vis[:, i, T - 1] = True
        elif kind == "some of the later":
            vis[:, i, 32:] = rng.random((B, T - 32)) < 0.3
        else:                                                                # every third row sees nothing, the others single nodes of one word
            if i % 3:
                vis[:, i, 32 * (i % ((T + 31) // 32)):32 * (i % ((T + 31) // 32)) + 32][:, ::7] = True
    return vis


@pytest.mark.parametrize("hq,hkv,d,T", [(2, 2, 128, 128), (2, 2, 64, 128), (8, 4, 64, 50), (16, 2, 128, 64), (8, 1, 64, 97), (12, 4, 128, 100)])
@pytest.mark.parametrize("kind", ["itself", "the last", "some of the later", "words"])
@pytest.mark.parametrize("shift", [0.0, -300.0, 300.0])
@pytest.mark.parametrize("flags", [0, 2])
def test_rows_that_name_none_of_the_first_nodes(hq, hkv, d, T, kind, shift, flags):
    """With no context, so that a tree's own tile is all there is, with so much that it is the second, third or ninth, and with scores about 0, far below and far above."""
    ctx = [0, 5, 130, 1000, 0]
    n = [T, T, T - 1, T, 40]
    c, q, kt, vt, vis, words, dn = _tree_case(hq, hkv, d, T, n, ctx, seed=T + d, vis=_masks(kind, len(ctx), T))
    if shift:                                                                # one dimension gives all of the nodes' scores a common part
        q[..., 0] = 16.0
        kt[..., 0] = shift / 16.0 * d ** 0.5
    lists = random_lists(c.ctx, hkv, 9, 64, seed=1)
    for hints in (True, False):
        out, lse, st = _run_tree(c, q, kt, vt, words, dn, lists, 64, flags, hints)
        assert st == OK
        _compare_tree(out, lse, q, c, kt, vt, vis, n, lists, 64, d ** -0.5)


@pytest.mark.parametrize("G,hkv,T", [(1, 3, 128), (8, 2, 64)])
def test_many_trees_whose_tiles_are_shared(G, hkv, T):
    """Enough key tiles that units are cut anywhere: a CTA's part may be the tree's own tile alone."""
    rng = np.random.default_rng(G)
    ctx = rng.integers(0, 3000, 60)
    n = rng.integers(33, T + 1, 60)
    c, q, kt, vt, vis, words, dn = _tree_case(G * hkv, hkv, 64, T, n, ctx, seed=G, vis=_masks("itself", 60, T))
    lists = random_lists(c.ctx, hkv, 20, 64, seed=2)
    out, lse, st = _run_tree(c, q, kt, vt, words, dn, lists, 64)
    assert st == OK
    _compare_tree(out, lse, q, c, kt, vt, vis, n, lists, 64, 0.125)
