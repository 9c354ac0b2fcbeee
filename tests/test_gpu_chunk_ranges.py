"""Ranges of packed rows that hold no row at all are reported, by every call that takes them, and every row stays as it was."""
import pytest
import torch

from tests.operator_refs import Paged, context, cuda

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
N = 11
# starts of three sequences: behind the last row, before the first one, both, a range that runs backwards
OUTSIDE = [([50, 60, 60, 60], []), ([12, 12, 13, 13], []), ([-9, -4, -4, -4], []), ([-9, -4, 0, 3], [0, 1, 2]), ([0, 3, 3, -2], [0, 1, 2])]
# empty ranges, wherever they lie, are no error
EMPTY = [([50, 50, 50, 50], []), ([-3, -3, -3, -3], []), ([0, 3, 3, 3], [0, 1, 2]), ([11, 11, 11, 11], [])]


def _case(flags=0):
    c = Paged([3, 4, 4], [5, 20, 0], 2, 64)
    x = torch.randn(N, 8, 64, generator=c.g, device="cuda", dtype=BF)
    return c, x[:, :4].contiguous(), x[:, 4:6], x[:, 6:], context(batch=3, n_q_heads=4, n_kv_heads=2, head_dim=64, flags=flags)


def _status(bad):
    from paper_2511_21699_b200 import _lib
    return _lib.CB_ERR_INVALID_ARG if bad else 0


@pytest.mark.parametrize("start,rows,bad", [(s, r, True) for s, r in OUTSIDE] + [(s, r, False) for s, r in EMPTY])
def test_append(start, rows, bad):
    c, q, k, v, cb = _case()
    out, kp, vp = torch.full_like(q, 7.0), c.k.clone(), c.v.clone()
    cb.cb_chunk_append(q, k, v, cuda(start), c.d_ctx, kp, vp, c.block_table, q_out=out)
    assert cb.cb_poll_status()[0] == _status(bad)
    rest = [r for r in range(N) if r not in rows]
    assert bool((out[rest] == 7).all()) and torch.equal(out[rows], q[rows])
    assert int((vp != c.v).flatten(2).any(-1).sum()) == len(rows)


def test_append_finds_the_bad_range_among_many():
    """The last of 2,000 sequences starts behind the rows; 1,999 have none, or one each."""
    c = Paged([1] * 2000, [3] * 2000, 2, 64)
    cb = context(batch=2000, n_q_heads=2, n_kv_heads=2, head_dim=64)
    q = torch.randn(500, 2, 64, generator=c.g, device="cuda", dtype=BF)
    start = [min(b, 500) for b in range(1999)] + [500, 500]
    for last, bad in ((500, False), (501, True)):
        start[-1] = last
        kp, vp, out = c.k.clone(), c.v.clone(), torch.empty_like(q)
        cb.cb_chunk_append(q, q, q, cuda(start), c.d_ctx, kp, vp, c.block_table, q_out=out)
        assert cb.cb_poll_status()[0] == _status(bad)
        assert torch.equal(out, q) and int((vp != c.v).flatten(2).any(-1).sum()) == 500


@pytest.mark.parametrize("flags", [0, 2])
@pytest.mark.parametrize("start,rows,bad", [(s, r, True) for s, r in OUTSIDE] + [(s, r, False) for s, r in EMPTY])
def test_attention(start, rows, bad, flags):
    c, q, _, _, cb = _case(flags)
    out, lse = torch.full_like(q, 7.0), torch.full((N, 4), 7.0, device="cuda")
    cb.cb_chunk_attn(q, c.k, c.v, c.block_table, cuda(start), c.d_ctx, out=out, lse=lse)
    assert cb.cb_poll_status()[0] == _status(bad)
    rest = [r for r in range(N) if r not in rows]
    assert bool((out[rest] == 7).all()) and bool((lse[rest] == 7).all())
    assert not rows or not bool((lse[rows] == 7).any())
