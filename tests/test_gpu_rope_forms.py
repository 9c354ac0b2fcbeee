"""Every form of the rotation kernel: chunk and tree, both head sizes, halves and neighbours, one to four groups of heads a warp, with head counts that
leave the last warp of a row part of its groups, against the formula in 64 bits."""
import numpy as np
import pytest
import torch

from tests.operator_refs import PAGE, Paged, context, cuda, rope_table
from tests.test_gpu_rope import _check, _norms, _rows

pytestmark = pytest.mark.gpu


def _groups(rows, hq, hkv, d):
    """Groups of heads that a warp holds side by side; from 8,000 on a warp takes two, from 28,000 on three (chunks); trees
    of 128 dims whose heads fill four take four from 100,000 on."""
    return rows * -(-(hq + 2 * hkv) // (512 // d))


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("hq,hkv,d,rot,norm,rows,lo,hi", [
    (12, 4, 128, 128, True, 300, 0, 8000), (9, 3, 64, 48, False, 300, 0, 8000),
    (36, 12, 128, 96, True, 701, 8000, 28000), (28, 4, 64, 64, True, 2003, 8000, 28000),
    (64, 8, 128, 128, True, 2100, 40000, 10 ** 9), (40, 40, 128, 64, False, 1400, 40000, 10 ** 9), (28, 4, 64, 64, True, 8203, 40000, 10 ** 9),
    (64, 8, 64, 32, False, 4100, 40000, 10 ** 9)])
def test_append_forms(hq, hkv, d, rot, norm, rows, lo, hi, inter):
    assert lo <= _groups(rows, hq, hkv, d) < hi
    new, ctx = [rows - rows // 3, 0, rows // 3], [5, 8, 100]
    c = Paged(new, ctx, hkv, d, seed=rows)
    x = _rows(rows, hq + 2 * hkv, d, c.g)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    table = rope_table(rows + 101, rot)
    wq, wk = _norms(d, c.g, norm)
    cb = context(batch=3, n_q_heads=hq, n_kv_heads=hkv, head_dim=d)
    kp, vp = c.k.clone(), c.v.clone()
    out = cb.cb_chunk_append(q, k, v, c.d_start, c.d_ctx, kp, vp, c.block_table, rope=table, q_norm=wq, k_norm=wk, interleaved=inter)
    assert cb.cb_poll_status()[0] == 0
    pos = cuda(np.concatenate([np.arange(a, a + m) for a, m in zip(ctx, new)]), torch.int64)
    _check(out, q, wq, 1e-6, table, pos, inter, "q")
    at = torch.cat([c.slots(b, ctx[b], ctx[b] + new[b]) for b in range(3)])
    _check(kp.view(-1, hkv, d)[at], k, wk, 1e-6, table, pos, inter, "k")
    assert torch.equal(vp.view(-1, hkv, d)[at], v)
    rest = torch.ones(kp.shape[0] * PAGE, dtype=torch.bool, device="cuda")
    rest[at] = False
    for got, was in ((kp, c.k), (vp, c.v)):
        assert torch.equal(got.view(-1, hkv, d)[rest], was.view(-1, hkv, d)[rest])


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("hq,hkv,d,rot,norm,B,T,lo,hi", [
    (12, 4, 128, 128, True, 5, 61, 0, 8000), (9, 3, 64, 48, False, 5, 61, 0, 8000),
    (36, 12, 128, 96, True, 11, 64, 8000, 28000), (28, 4, 64, 64, True, 33, 61, 8000, 28000),
    (66, 11, 128, 128, True, 16, 128, 40000, 10 ** 9), (64, 8, 128, 32, False, 33, 64, 40000, 10 ** 9), (28, 4, 64, 64, True, 70, 121, 40000, 10 ** 9),
    (64, 8, 64, 64, False, 40, 128, 40000, 10 ** 9),
    (64, 8, 128, 128, True, 40, 128, 100000, 10 ** 9), (24, 4, 128, 64, False, 98, 128, 100000, 10 ** 9)])
def test_tree_forms(hq, hkv, d, rot, norm, B, T, lo, hi, inter):
    assert lo <= _groups(B * T, hq, hkv, d) < hi
    rng = np.random.default_rng(T)
    g = torch.Generator(device="cuda").manual_seed(B)
    n = rng.integers(0, T + 1, B)
    n[0] = T
    dep = rng.integers(0, 9, (B, T))
    dep[np.arange(T)[None] >= n[:, None]] = -1
    ctx = rng.integers(0, 900, B)
    x = _rows(B * T, hq + 2 * hkv, d, g)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    table = rope_table(910, rot)
    wq, wk = _norms(d, g, norm)
    cb = context(batch=B, max_nodes=T, n_q_heads=hq, n_kv_heads=hkv, head_dim=d)
    got = cb.cb_tree_rope(q, k, v, dict(depth=cuda(dep), n_nodes=cuda(n)), cuda(ctx), rope=table, q_norm=wq, k_norm=wk, interleaved=inter)
    assert cb.cb_poll_status()[0] == 0
    live = cuda(np.arange(T)[None] < n[:, None], torch.bool).view(-1)
    pos = cuda((ctx[:, None] + dep).clip(0).reshape(-1), torch.int64)[live]
    for a, y, w in zip((q, k), got, (wq, wk)):
        y = y.view(B * T, -1, d)
        _check(y[live], a[live], w, 1e-6, table, pos, inter, "tree")
        assert bool((y[~live] == 0).all())
    y = got[2].view(B * T, -1, d)
    assert torch.equal(y[live], v[live]) and bool((y[~live] == 0).all())
