"""cb_chunk_attn's scale: zero selects 1 / sqrt(head_dim), positive ones are taken, everything else is refused and nothing is written."""
import math

import pytest
import torch

from tests.operator_refs import Paged, attention, context, cuda, F8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("flags", [0, 2])
def test_scale(flags):
    from paper_2511_21699_b200 import CachebackError
    c = Paged([5], [30], 1, 64)
    q = torch.randn(5, 2, 64, generator=c.g, device="cuda", dtype=torch.bfloat16)
    cb = context(n_q_heads=2, n_kv_heads=1, head_dim=64, flags=flags)
    at = c.slots(0, 0, 35)
    for scale, used in ((0.0, 0.125), (0.125, 0.125), (0.5, 0.5), (1e-3, 1e-3)):
        out = cb.cb_chunk_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, scale=scale)
        ref, _, bound, _ = attention(q, c.k.view(-1, 1, 64)[at], c.v.view(-1, 1, 64)[at], 30, used)
        assert bool(((out.to(F8) - ref).abs() <= bound).all()), scale
    out = torch.full_like(q, 7.0)
    for scale in (-0.125, -1e-30, math.nan, math.inf, -math.inf):
        with pytest.raises(CachebackError, match="invalid argument"):
            cb.cb_chunk_attn(q, c.k, c.v, c.block_table, c.d_start, c.d_ctx, out=out, scale=scale)
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and cb.cb_poll_status()[0] == 0
