"""cb_block_select by the C interface: numbers at the ends of their types."""
import ctypes as C

import pytest
import torch

from paper_2511_21699_b200 import _lib
from tests.operator_refs import context

pytestmark = pytest.mark.gpu
LEAST, MOST = -(1 << 31), (1 << 31) - 1


@pytest.mark.parametrize("select,first,last", [(LEAST, 0, 1), (LEAST, MOST, 1), (LEAST + 3, 0, 10), (LEAST, 0, MOST), (-1, 0, 1), (-1, 0, MOST), (0, 0, 1), (MOST, 0, 1), (4, MOST, 1), (4, 0, MOST), (4, LEAST, 1),
                                               (4, 0, LEAST), (4, MOST, MOST), (1025, 0, 1), (4, 4, 1)])
def test_lists_of_impossible_length(select, first, last):
    cb = context(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, max_nodes=8)
    lib = _lib.load()
    base = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda").data_ptr()
    before = cb.launch_count()
    a = _lib.CbBlockSelectArgsC(base, base, None, base, base, base, base, base, 5, 9, 18, 64, select, first, last, 0, 0)
    assert lib.cb_block_select(cb._h, C.byref(a), None) == _lib.CB_ERR_INVALID_ARG
    assert cb.launch_count() == before


@pytest.mark.parametrize("G,most", [(15, 20452225), (12, 44739242), (7, 204522252)])
def test_chunks_of_more_rows_than_can_be_told_apart(G, most):
    """Row and head of a query come from a product that is exact up to there; the sequence behind is turned away before its queries are read."""
    cb = context(batch=2, n_q_heads=G, n_kv_heads=1, head_dim=64)
    q = torch.zeros(2, G, 64, dtype=torch.bfloat16, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    start, ctx, table = i32(0, 2, 2 + most + 1), i32(640, 640), torch.zeros(2, 40, dtype=torch.int32, device="cuda")
    mean, scale = torch.zeros(1, 1, 64, dtype=torch.int8, device="cuda"), torch.zeros(1, 1, device="cuda")
    out = torch.full((2, 1, 4), 77, dtype=torch.int32, device="cuda")
    a = _lib.CbBlockSelectArgsC(q.data_ptr(), start.data_ptr(), None, mean.data_ptr(), scale.data_ptr(), table.data_ptr(), ctx.data_ptr(), out.data_ptr(), MOST, 40, 1, 64, 4, 1, 2, 0, 0)
    assert _lib.load().cb_block_select(cb._h, C.byref(a), None) == 0
    assert cb.cb_poll_status()[0] == _lib.CB_ERR_INVALID_ARG
    assert out.cpu().tolist() == [[[0, 1, 8, 9]], [[-1] * 4]]
