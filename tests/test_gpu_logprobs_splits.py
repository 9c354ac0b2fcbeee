"""Rows on both sides of where a row is shared by more CTAs: equal results whatever the split, against the formulas in 64 bits."""
import pytest
import torch

from tests.operator_refs import F8, context, cuda, likelihoods

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [0, 3, 32])
@pytest.mark.parametrize("V", [15999, 23999, 24000, 24001, 32000, 33001, 47999, 48000, 64003])
def test_around_the_bounds(V, top, dtype):
    cb = context(vocab=V)
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (torch.randn(160, V, generator=g, device="cuda") * (0.3 + 3 * torch.rand(160, 1, generator=g, device="cuda"))).to(dtype)
    x[:, ::7] = -float("inf")
    tok = torch.randint(V // 7, (160,), generator=g, device="cuda", dtype=torch.int32) * 7 + 1
    ref, bound = likelihoods(x, tok, top)
    for n in (1, 20, 41, 75, 160):
        got = cb.cb_logprobs(x[:n], tok[:n], top_k=top)
        for k, want in ref.items():
            fine = got[k].long() == want[:n] if k == "top_ids" else (got[k].to(F8) - want[:n]).abs() <= bound[k][:n]
            assert bool(fine.all()), (n, k)
    assert cb.cb_poll_status()[0] == 0
