"""cb_logprobs on finite logits whose differences leave fp32, rows of one CTA and rows that a cluster shares."""
import math

import pytest
import torch

from tests.operator_refs import F8, context, cuda, likelihoods

pytestmark = pytest.mark.gpu


def check_beyond_range(got, x, tok, top, rows=slice(None)):
    """As the definition in 64 bits, put into fp32 (what lies below its range is -inf there), within the bounds of the sums."""
    ref, bound = likelihoods(x, tok, top)
    for k in ("logprobs", "entropy", "top_logprobs"):
        a, b = got[k][rows], ref[k][rows]
        fine = (a == b.float()) | ((a.to(F8) - b).abs() <= bound[k][rows])
        assert bool(fine.all()), (k, a, b)
    assert torch.equal(got["top_ids"][rows].long(), ref["top_ids"][rows])


@pytest.mark.parametrize("V", [11, 4099, 128256])             # less than a step of a thread, a CTA's, a cluster's
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_finite_logits_further_apart_than_fp32_holds(V, dtype):
    cb = context(vocab=V)
    low, at = torch.finfo(dtype).min, V // 2
    x = torch.full((7, V), -2e38, device="cuda")
    x[0, at] = 2e38                                           # the difference is -4e38
    x[1, 1] = x[1, V - 2] = 2e38                              # two of them: log 2
    x[2] = low                                                # a mask of the type's lowest value beside large logits
    x[2, at:at + 3] = 1e37
    x[3] = low
    x[3, :4] = -low
    x[4] = (torch.arange(V, device="cuda") / (V - 1) * 2 - 1) * 3e38      # (a linspace would form 6e38)
    x[5, at] = 2e38
    x[5, ::3] = -math.inf                                     # forbidden ones among them
    x[5, at] = 2e38
    x[6] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 3e38, -3e38)
    x = x.to(dtype)
    assert not bool(x.isnan().any()) and not bool((x == math.inf).any())
    tok = cuda([at, 1, at + 1, 0, V - 1, at, V - 1])
    got = cb.cb_logprobs(x, tok, top_k=9)
    check_beyond_range(got, x, tok, 9)
    assert bool((got["entropy"] >= 0).all()) and cb.cb_poll_status()[0] == 0
