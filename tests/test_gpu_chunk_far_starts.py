"""Starts at the ends of the 32-bit range: the sequence is reported and its rows stay as they were."""
import pytest
import torch

from tests.operator_refs import Paged, context, cuda

pytestmark = pytest.mark.gpu
LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("call", ["append", "attention", "attention on CUDA cores"])
@pytest.mark.parametrize("start,live", [([LOW, 5, 9], range(5, 9)), ([LOW, LOW + 1, 9], []), ([0, 4, HIGH], range(4)), ([LOW, 0, HIGH], []), ([LOW, HIGH, HIGH], [])])
def test_far_starts(call, start, live):
    from paper_2511_21699_b200 import _lib
    c = Paged([9, 9], [3, 40], 1, 64)
    q = torch.randn(9, 2, 64, generator=c.g, device="cuda", dtype=torch.bfloat16)
    k = torch.randn(9, 1, 64, generator=c.g, device="cuda", dtype=torch.bfloat16)
    cb = context(batch=2, n_q_heads=2, n_kv_heads=1, head_dim=64, flags=2 if "CUDA" in call else 0)
    out, lse, kp, vp = torch.full_like(q, 7.0), torch.full((9, 2), 7.0, device="cuda"), c.k.clone(), c.v.clone()
    if call == "append":
        cb.cb_chunk_append(q, k, k, cuda(start), c.d_ctx, kp, vp, c.block_table, q_out=out)
        assert int((vp != c.v).flatten(2).any(-1).sum()) == len(live)
    else:
        cb.cb_chunk_attn(q, c.k, c.v, c.block_table, cuda(start), c.d_ctx, out=out, lse=lse)
        assert bool((lse[[r for r in range(9) if r not in live]] == 7).all())
    assert cb.cb_poll_status()[0] == _lib.CB_ERR_INVALID_ARG
    rest = [r for r in range(9) if r not in live]
    assert bool((out[rest] == 7).all()) and not bool((out[list(live)] == 7).any())
