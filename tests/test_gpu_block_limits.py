"""cb_block_select by the C interface: numbers at the ends of their types are refused before anything is launched."""
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
