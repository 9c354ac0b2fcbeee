"""Calls on a stream other than the current one that are given no tensors for their results: what they make must not lie in memory that work queued on the current stream still
uses, nor be handed out again before it is done with."""
import ctypes as C

import pytest
import torch

from tests.block_refs import random_lists
from tests.operator_refs import Paged, context, cuda

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
PAUSE = 100_000_000                                                          # cycles: some 50 ms


class _Raw:
    """A stream of which only the handle is known."""
    def __init__(self, stream):
        self.cuda_stream = stream.cuda_stream


@pytest.fixture(scope="module")
def calls():
    c = Paged([3, 40], [700, 90], 2, 64)
    T = 8
    cb = context(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, max_nodes=T, vocab=50)
    q = torch.randn(43, 8, 64, device="cuda", generator=c.g).to(BF)
    qt, kt = torch.randn(2, T, 8, 64, device="cuda", generator=c.g).to(BF), torch.randn(2, T, 2, 64, device="cuda", generator=c.g).to(BF)
    mean, scale = cb.alloc_summary(c.num_pages)
    cb.cb_block_summary(c.k, c.block_table, cuda([0, 0]), c.d_ctx, mean, scale, block=32)
    lists = cuda(random_lists(c.ctx, 2, 4, 32, seed=0))
    mask, n = torch.ones(2, T, 1, dtype=torch.int32, device="cuda"), cuda([T, T])
    logits, tok = torch.randn(43, 50, device="cuda", generator=c.g), torch.zeros(43, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    keep = (c, cb)
    return keep, {
        "cb_slot_map": lambda s: cb.cb_slot_map(c.d_start, c.d_ctx, c.block_table, c.num_pages, 43, stream=s),
        "cb_block_select": lambda s: cb.cb_block_select(q, mean, scale, c.block_table, c.d_ctx, q_start=c.d_start, block=32, n_select=4, stream=s),
        "cb_block_attn": lambda s: cb.cb_block_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, lists, block=32, stream=s),
        "cb_block_tree_attn": lambda s: cb.cb_block_tree_attn(qt, c.k, c.v, c.block_table, c.d_ctx, kt, kt, mask, n, lists, block=32, stream=s),
        "cb_chunk_attn": lambda s: cb.cb_chunk_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, stream=s),
        "cb_tree_attn": lambda s: cb.cb_tree_attn(qt, c.k, c.v, c.block_table, c.d_ctx, kt, kt, mask, n, stream=s),
        "cb_logprobs": lambda s: cb.cb_logprobs(logits, tok, top_k=3, stream=s),
    }


def _tensors(res):
    return list(res.values()) if isinstance(res, dict) else [res]


NAMES = ["cb_slot_map", "cb_block_select", "cb_block_attn", "cb_block_tree_attn", "cb_chunk_attn", "cb_tree_attn", "cb_logprobs"]


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_reads(calls, name, raw):
    call = calls[1][name]
    want = [t.clone() for t in _tensors(call(None))]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    held = [[torch.full_like(t, 3) for _ in range(4)] for t in want]
    copies = [[torch.empty_like(t) for _ in range(4)] for t in want]
    torch.cuda.synchronize()
    torch.cuda._sleep(PAUSE)
    for x, y in zip(held, copies):
        for a, b in zip(x, y):
            b.copy_(a)                                                       # queued behind the pause
    del held, x, a                                                           # free, for the current stream
    got = _tensors(call(_Raw(side) if raw else side))
    torch.cuda.synchronize()
    for y in copies:
        for b in y:
            assert bool((b == 3).all())
    for g, w in zip(got, want):
        assert torch.equal(g, w)


@pytest.mark.parametrize("name", NAMES)
def test_results_that_the_current_stream_still_reads(calls, name):
    """Freed while a copy on the current stream is queued behind a pause: the next call on the side stream gets other memory."""
    call = calls[1][name]
    side = torch.cuda.Stream()
    got = _tensors(call(side))
    side.synchronize()
    want = [t.clone() for t in got]
    copies = [torch.empty_like(t) for t in got]
    torch.cuda.synchronize()
    torch.cuda._sleep(PAUSE)
    for a, b in zip(got, copies):
        b.copy_(a)
    shapes = [(t.shape, t.dtype) for t in got]
    del got, a
    with torch.cuda.stream(side):
        other = [torch.zeros(s, dtype=t, device="cuda") for s, t in shapes for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(b, w) for b, w in zip(copies, want)) and len(other) == 3 * len(shapes)
