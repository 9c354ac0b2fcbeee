"""cb_logprobs on rows without a value: NaN, +inf or no finite logit gives NaN in every number of the row, the alternatives' among them,
whichever and however many of its elements are NaN; rows of one CTA and rows that a cluster shares."""
import math

import pytest
import torch

from tests.operator_refs import context, cuda, likelihoods, F8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [3, 40, 3001, 128256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [0, 2, 32])
def test_rows_without_a_value(V, dtype, top):
    cb = context(vocab=V)
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(8, V, generator=g, device="cuda")
    x[0] = math.nan
    x[1, V // 2] = math.nan
    x[2, :] = -math.inf
    x[3, V - 1] = math.inf
    x[4, 1:] = math.nan                                       # one element that is a number, and the lowest
    x[4, 0] = torch.finfo(dtype).min
    x[5] = -math.inf
    x[5, V - 1] = math.nan
    x[6] = math.inf
    x = x.to(dtype)
    tok = cuda([0, 1, 2, 0, 0, 1, 2, 1])
    got = cb.cb_logprobs(x, tok, top_k=top)
    assert cb.cb_poll_status()[0] == 0
    assert bool(got["logprobs"][:7].isnan().all()) and bool(got["entropy"][:7].isnan().all())
    ref, bound = likelihoods(x[7:], tok[7:], top)             # its neighbour in the batch
    assert bool(((got["logprobs"][7:].to(F8) - ref["logprobs"]).abs() <= bound["logprobs"]).all())
    if not top:
        return
    k = min(top, V)                                           # places that the vocabulary fills
    assert bool(got["top_logprobs"][:7, :k].isnan().all())
    assert bool((got["top_logprobs"][:, k:] == -math.inf).all()) and bool((got["top_ids"][:, k:] == -1).all())
    ids = got["top_ids"][:7, :k]
    assert bool(((ids >= -1) & (ids < V)).all()) and bool((ids[0] == -1).all())     # a NaN is nobody's alternative
    assert ids[4].tolist() == [0] + [-1] * (k - 1) and int(ids[3, 0]) == V - 1 and ids[2].tolist() == list(range(k)) and ids[6].tolist() == list(range(k))
    assert torch.equal(got["top_ids"][7, :k].long(), ref["top_ids"][0])
