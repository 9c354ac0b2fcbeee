"""What the calls that keep a cache's tables and attend to selected blocks refuse.  Nothing here reaches a GPU."""
import ctypes as C

import pytest
import torch

import __graft_entry__
from paper_2511_21699_b200 import _lib, api


@pytest.fixture(scope="module")
def host():
    __graft_entry__.build()
    return api._host()


class _Stream:
    cuda_stream = 0


SHAPE = (0, 2, 4, 4, 2, 64, 16, 3, 10)                                       # device, batch, nodes, heads, kv heads, dims, page, depth, vocabulary


def test_no_context(host):
    lib = _lib.load()
    p = 1 << 20                                                              # (not looked at)
    args = {"cb_slot_map": _lib.CbSlotMapArgsC, "cb_block_summary": _lib.CbBlockSummaryArgsC, "cb_block_select": _lib.CbBlockSelectArgsC}
    for name, t in args.items():
        assert getattr(lib, name)(None, C.byref(t()), None) == _lib.CB_ERR_INVALID_ARG
    assert lib.cb_pages_assign(None, p, p, 1, p, p, 1, p, None) == _lib.CB_ERR_INVALID_ARG
    assert lib.cb_block_attn(None, C.byref(_lib.CbChunkAttnArgsC()), p, 64, 4, None) == _lib.CB_ERR_INVALID_ARG
    assert lib.cb_block_tree_attn(None, C.byref(_lib.CbAttnArgsC()), p, 64, 4, None) == _lib.CB_ERR_INVALID_ARG


def test_tensors_that_are_no_cuda_tensors(host):
    h, s = C.c_void_p(None), _Stream()
    i = torch.zeros(2, 4, dtype=torch.int32)
    for call in (lambda x: host.pages_assign(h, SHAPE, x, i, i, i, i, s), lambda x: host.slot_map(h, SHAPE, x, i, i, 4, 4, {}, s),
                 lambda x: host.block_summary(h, SHAPE, x, i, i, i, i, i, 64, s), lambda x: host.block_select(h, SHAPE, x.view(1, 2, 4) if x is i else x, i, i, i, i, i, None, 64, 4, 1, 1, 0, 0, i, s),
                 lambda x: host.block_tree_attn(h, SHAPE, x, i, i, i, i, i, i, i, i, i, None, 0, 0.0, i, 64, s)):
        for bad in (i, [1, 2], "x", 3, None):
            with pytest.raises((api.CachebackError, TypeError, AttributeError), match="expected a contiguous CUDA tensor|view"):
                call(bad)


def test_rows_of_either_kind_but_not_both(host):
    h, i = C.c_void_p(None), torch.zeros(3, dtype=torch.int32)
    for q_start, n in ((None, None), (i, i)):
        with pytest.raises(api.CachebackError, match="q_start or n_nodes must be given, one of the two"):
            host.block_select(h, SHAPE, i, i, i, i, i, q_start, n, 64, 4, 1, 1, 0, 0, i, _Stream())


def test_numbers_of_arguments(host):
    for name in ("pages_assign", "slot_map", "block_summary", "block_select", "block_attn", "block_tree_attn"):
        with pytest.raises(TypeError, match="expected .* arguments"):
            getattr(host, name)(C.c_void_p(None), SHAPE)
