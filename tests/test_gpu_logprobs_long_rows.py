"""The search for the alternatives in rows so long that a noted maximum covers several steps of a thread: large elements in the last, partial slot, in
every step of a slot, in many slots, more equals than places.  (A step is 256 threads x 4 pieces of 16 bytes, a thread notes 32 maxima.)"""
import math

import pytest
import torch

from tests.operator_refs import cuda, context, likelihoods, F8

pytestmark = pytest.mark.gpu
STEP, SLOTS = 256 * 4, 32


def _split(V, E, cs):
    """Steps of a CTA that has the first of cs parts of a row, and how many of them a noted maximum covers."""
    per = -(-(V // E) // cs)
    steps = -(-per // STEP)
    return per, steps, -(-steps // SLOTS)


def _rows(V, n, dtype, cs, g):
    """Rows 0..5 with the large elements where the search has to look; the others random."""
    E = 8 if dtype == torch.bfloat16 else 4
    per, steps, covered = _split(V, E, cs)
    x = torch.randn(n, V, generator=g, device="cuda")
    step_of = torch.arange(V // E * E, device="cuda") // E % per // STEP      # of every element, in its part
    last = step_of >= (steps - 1) // covered * covered        # the last slot's: fewer steps than the others
    pick = lambda mask, k: mask.nonzero()[:, 0][torch.randperm(int(mask.sum()), generator=g, device="cuda")[:k]]
    x[0, pick(last, 40)] += 20                                # all alternatives in the last slot
    for s in range(covered):                                  # one thread's elements of each step of one slot
        at = (2 * covered + s) * STEP * E + 77 * E
        x[1, at:at + E] = 15 + s + torch.arange(E, device="cuda") / 4
    x[2, pick(step_of % covered == covered - 1, 600)] += 9    # many, in the last step of their slots
    x[3] = x[3].clamp(max=2.0)                                # thousands of equals at the top
    x[4] = -math.inf
    x[4, pick(step_of >= 0, 7)] = 0.5                         # fewer tokens than alternatives
    x[5] = torch.arange(V, device="cuda") / V * 30
    return x.to(dtype)


def _check(V, n, dtype, cs, top):
    cb = context(vocab=V)
    g = torch.Generator(device="cuda").manual_seed(V)
    x = _rows(V, n, dtype, cs, g)
    tok = x[:, :V].argmax(1).to(torch.int32)
    got = cb.cb_logprobs(x, tok, top_k=top)
    assert cb.cb_poll_status()[0] == 0
    for i in range(0, n, 16):
        ref, bound = likelihoods(x[i:i + 16], tok[i:i + 16], top)
        for k, want in ref.items():
            a = got[k][i:i + 16]
            fine = a.long() == want if k == "top_ids" else (a == want) | ((a.to(F8) - want).abs() <= bound[k])
            assert bool(fine.all()), (k, i)


@pytest.mark.parametrize("dtype,V", [(torch.float32, 1200007), (torch.bfloat16, 2400011)])
@pytest.mark.parametrize("n", [6, 40, 90, 200, 330])
def test_slots_of_several_steps_whatever_the_split(dtype, V, n):
    """However many CTAs up to eight share a row, each has more steps than a thread notes maxima."""
    E = 8 if dtype == torch.bfloat16 else 4
    for cs in (1, 2, 4, 8):
        assert _split(V, E, cs)[2] > 1
    for cs in (1, 8) if n == 6 else (1,):                     # where in its part an element lies, for either split
        _check(V, n, dtype, cs, 20)


@pytest.mark.parametrize("dtype,V", [(torch.float32, 151936), (torch.float32, 140001), (torch.bfloat16, 280003)])
def test_many_rows_of_a_long_vocabulary(dtype, V):
    """A row per CTA, with 35 and 38 steps: one slot of one step, or none."""
    assert _split(V, 8 if dtype == torch.bfloat16 else 4, 1)[2] == 2
    _check(V, 320, dtype, 1, 20)
