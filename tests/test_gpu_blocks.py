"""cb_block_summary and cb_block_select: whole numbers, all equal to plain references in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests.block_refs import select, summary
from tests.operator_refs import F8, PAGE, Paged, context, cuda

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
OK, INVALID, FULL = 0, 1, 8


def _summarise(c, cb, lo, hi, block, mean=None, scale=None):
    pages, _, hkv, d = c.k.shape
    mean = torch.full((pages, hkv, d), 99, device="cuda", dtype=torch.int8) if mean is None else mean
    scale = torch.full((pages, hkv), -5.0, device="cuda") if scale is None else scale
    cb.cb_block_summary(c.k, c.block_table, cuda(lo), cuda(hi), mean, scale, block=block)
    return mean, scale, cb.cb_poll_status()[0]


def _check_summary(c, lo, hi, block, mean, scale, skip=()):
    """Touched blocks hold their summaries, nothing else is written."""
    ref_m, ref_s = torch.full_like(mean, 99), torch.full_like(scale, -5.0).to(F8)
    flat = c.k.view(-1, *c.k.shape[2:])
    for b in range(len(lo)):
        if b in skip or lo[b] >= hi[b]:
            continue
        for j in range(lo[b] // block, -(-hi[b] // block)):
            m, s = summary(flat[c.slots(b, j * block, min((j + 1) * block, hi[b]))])
            at = c.bt[b, j * block // PAGE]
            ref_m[at], ref_s[at] = m.to(torch.int8), s
    assert torch.equal(mean, ref_m)
    # the scale: a division and a rounding in 64 bits, one to fp32
    assert bool(((scale.to(F8) - ref_s).abs() <= ref_s.abs() * 2.0 ** -24 * 1.001).all())


@pytest.mark.parametrize("hkv,d", [(1, 64), (2, 128), (3, 64), (5, 128), (8, 128), (9, 64), (40, 128)])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_summaries(hkv, d, block):
    lens = np.array([0, 1, 15, 16, 17, 127, 128, 129, 200, 1000])
    c = Paged(lens, np.zeros_like(lens), hkv, d, seed=block + hkv)
    c.k += torch.randn(c.num_pages, 1, hkv, d, generator=c.g, device="cuda", dtype=BF)
    cb = context(batch=len(lens), n_q_heads=hkv, n_kv_heads=hkv, head_dim=d)
    for lo in (np.zeros_like(lens), np.maximum(lens - 1, 0), lens, np.maximum(lens - 40, 0), lens + 3):
        mean, scale, st = _summarise(c, cb, lo, lens, block)
        assert st == OK
        _check_summary(c, lo, lens, block, mean, scale)


def test_summaries_of_many_sequences_and_one_long():
    lens = np.concatenate([np.full(300, 70), [9000], np.full(299, 33)])
    c = Paged(lens, np.zeros_like(lens), 2, 64)
    cb = context(batch=600, n_q_heads=2, n_kv_heads=2)
    lo = np.where(lens == 9000, 0, lens - 1)
    mean, scale, st = _summarise(c, cb, lo, lens, 64)
    assert st == OK
    _check_summary(c, lo, lens, 64, mean, scale)


def test_summary_token_by_token_is_the_summary_at_once():
    c = Paged([200], [0], 2, 128)
    cb = context(n_q_heads=2, n_kv_heads=2, head_dim=128)
    at_once = _summarise(c, cb, np.array([0]), np.array([200]), 64)[:2]
    m, s = (torch.full_like(x, 99 if x.dtype == torch.int8 else -5.0) for x in at_once)
    at = 0
    for step in (1, 1, 62, 1, 7, 60, 68):
        _summarise(c, cb, np.array([at]), np.array([at + step]), 64, m, s)
        at += step
    assert at == 200 and torch.equal(m, at_once[0]) and torch.equal(s, at_once[1])


def test_summary_of_extreme_keys():
    c = Paged([64] * 6, [0] * 6, 1, 64)
    c.k.zero_()
    at = lambda b: c.slots(b, 0, 64)
    flat = c.k.view(-1, 1, 64)
    flat[at(1)] = torch.finfo(BF).max
    flat[at(2)] = 2.0 ** -133                                                # the smallest bf16
    flat[at(3)[5]] = math.inf
    flat[at(4)[9], 0, 3] = math.nan
    flat[at(5)] = torch.cat((torch.full((32, 1, 64), 3e38), torch.full((32, 1, 64), -3e38))).to(BF).cuda()      # cancels: a sum in fp32 would overflow
    flat[at(5)[0], 0, 1] += 0
    flat[at(5)[0], 0, 2] = 1.0
    cb = context(batch=6)
    lens = np.full(6, 64)
    mean, scale, st = _summarise(c, cb, 0 * lens, lens, 64)
    first = c.bt[:, 0]
    m, s = mean[first][:, 0].cpu(), scale[first][:, 0].cpu()
    assert st == OK
    assert (m[0] == 0).all() and s[0] == 0
    assert (m[1] == 127).all() and math.isclose(float(s[1]), float(torch.finfo(BF).max) / 127, rel_tol=1e-6)
    assert (m[2] == 0).all()                                                 # below 1e-30 everything is nothing
    for b in (3, 4):
        assert (m[b] == 0).all() and s[b] == math.inf
    ref = summary(flat[at(5)])
    assert torch.equal(m[5].long(), ref[0][0].cpu())


def test_summary_refusals_on_the_device():
    lens = np.array([70, 130, 64, 20])
    c = Paged(lens, 0 * lens, 2, 64)
    cb = context(batch=4, n_q_heads=2, n_kv_heads=2)
    lo = np.array([0, -1, 0, 0])
    mean, scale, st = _summarise(c, cb, lo, lens, 64)
    assert st == INVALID
    _check_summary(c, lo, lens, 64, mean, scale, skip=(1,))
    hi = np.array([70, 130, 64, 16 * c.bt.shape[1] + 1])
    mean, scale, st = _summarise(c, cb, 0 * lens, hi, 64)
    assert st == FULL
    _check_summary(c, 0 * lens, hi, 64, mean, scale, skip=(3,))
    for bad in (-1, c.num_pages, 1 << 30):
        c.block_table[2, 1] = bad
        mean, scale, st = _summarise(c, cb, 0 * lens, lens, 64)
        assert st == INVALID
        _check_summary(c, 0 * lens, lens, 64, mean, scale, skip=(2,))


# ------------------------------------------------------------------------------------------------ selection
class Scored:
    """Random summaries of sequences with ctx tokens."""

    def __init__(self, ctx, hkv, d, block, seed=0, ties=False):
        self.ctx, self.block = np.asarray(ctx), block
        self.c = Paged(0 * self.ctx, self.ctx, 1, 64, seed=seed)             # (its keys are not used)
        g = self.c.g
        pages = self.c.num_pages
        self.mean = torch.randint(-127, 128, (pages, hkv, d), generator=g, device="cuda", dtype=torch.int8)
        self.scale = torch.rand(pages, hkv, generator=g, device="cuda") + 0.01
        if ties:                                                             # three kinds of blocks
            kind = torch.randint(3, (pages,), generator=g, device="cuda")
            self.mean, self.scale = self.mean[kind].contiguous(), self.scale[kind].contiguous()

    def first_pages(self, b):
        nb = -(-int(self.ctx[b]) // self.block)
        return cuda(self.c.bt[b, np.arange(nb) * self.block // PAGE], torch.int64)


def _select(s, q, K, nf=1, nl=2, q_start=None, n=None, hints=False, cb=None, T=1):
    hkv, d = s.mean.shape[1:]
    hq = q.shape[-2]
    cb = cb or context(batch=len(s.ctx), n_q_heads=hq, n_kv_heads=hkv, head_dim=d, max_nodes=T)
    out = torch.full((len(s.ctx), hkv, K), 55, device="cuda", dtype=torch.int32)
    rows = dict(q_start=cuda(q_start), max_chunk=int(np.diff(q_start).max()) if hints else 0) if n is None else dict(n_nodes=cuda(n))
    cb.cb_block_select(q, s.mean, s.scale, s.c.block_table, s.c.d_ctx, **rows, block=s.block, n_select=K, n_first=nf, n_last=nl,
                       max_ctx=int(s.ctx.max()) if hints else 0, blocks=out)
    return out.cpu().numpy(), cb.cb_poll_status()[0]


def _check_select(s, q, out, K, nf, nl, rows_of, skip=()):
    hkv, d = s.mean.shape[1:]
    G = q.shape[-2] // hkv
    for b in range(len(s.ctx)):
        at = s.first_pages(b)
        for h in range(hkv):
            votes = rows_of(b)[:, h * G:h * G + G].reshape(-1, d)
            ref = [] if b in skip else select(votes, s.mean[at, h], s.scale[at, h], K, nf, nl)
            assert out[b, h].tolist() == ref + [-1] * (K - len(ref)), (b, h, int(s.ctx[b]))


def _chunks(new, hq, d, g, scale=1.5):
    start = np.concatenate([[0], np.cumsum(new)])
    return start, (torch.randn(int(start[-1]), hq, d, generator=g, device="cuda") * scale).to(BF)


@pytest.mark.parametrize("hq,hkv,d,block,K,nf,nl,new,ctx", [
    (8, 8, 64, 64, 4, 1, 2, [1], [1000]),
    (32, 8, 128, 64, 32, 1, 2, [1] * 5, [0, 1, 2048, 2049, 32768]),
    (16, 4, 64, 16, 7, 0, 1, [1, 0, 3], [500, 900, 5003]),
    (28, 4, 128, 32, 40, 2, 5, [5, 40, 1], [3000, 4000, 1280]),
    (16, 1, 128, 128, 3, 1, 2, [9, 33, 2], [20000, 385, 384]),
    (40, 40, 128, 64, 8, 0, 8, [2, 1], [6000, 577]),
    (5, 1, 64, 16, 128, 64, 64, [130], [9000]),
    (16, 1, 64, 64, 33, 3, 3, [256, 1], [40000, 2200]),
    (2, 2, 64, 16, 1024, 1, 1, [3], [40000]),
    (4, 2, 128, 64, 1, 0, 1, [1], [640]),
])
def test_selection_of_chunks(hq, hkv, d, block, K, nf, nl, new, ctx):
    s = Scored(ctx, hkv, d, block, seed=K)
    start, q = _chunks(new, hq, d, s.c.g)
    for hints in (False, True):
        out, st = _select(s, q, K, nf, nl, q_start=start, hints=hints)
        assert st == OK
        _check_select(s, q, out, K, nf, nl, lambda b: q[start[b]:start[b + 1]])


@pytest.mark.parametrize("T,n", [(1, [1, 1, 0]), (64, [64, 17, 1]), (61, [61, 0, 33]), (128, [128, 127, 5])])
def test_selection_of_trees(T, n):
    s = Scored([9000, 3001, 700], 4, 64, 32, seed=T)
    q = torch.randn(3, T, 16, 64, generator=s.c.g, device="cuda").to(BF)
    out, st = _select(s, q, 20, n=np.array(n), T=T)
    assert st == OK
    _check_select(s, q, out, 20, 1, 2, lambda b: q[b, :n[b]])


@pytest.mark.parametrize("K", [3, 4, 17, 100])
def test_equal_scores_go_by_number(K):
    s = Scored([5000, 40000], 2, 64, 16, ties=True)
    start, q = _chunks([1, 3], 4, 64, s.c.g)
    out, st = _select(s, q, K, q_start=start)
    assert st == OK
    _check_select(s, q, out, K, 1, 2, lambda b: q[start[b]:start[b + 1]])
    q.zero_()                                                                # all scores zero
    out, st = _select(s, q, K, q_start=start)
    nb = [-(-5000 // 16), 2500]
    assert all(out[b, h].tolist() == list(range(K - 2)) + [nb[b] - 2, nb[b] - 1] for b in range(2) for h in range(2))


def test_scores_that_are_no_numbers_come_first_and_zero_scales_are_zero():
    s = Scored([6400], 1, 64, 64)
    at = s.first_pages(0)
    s.scale[at[[40, 60]]], s.mean[at[[40, 60]]] = math.inf, 0                # what a mean that is not finite leaves
    s.scale[at[10]] = math.nan
    s.scale[at[20:30]] = 0.0
    start, q = _chunks([1], 1, 64, s.c.g)
    for K in (4, 5, 6, 50, 95):
        out, st = _select(s, q, K, q_start=start)
        assert st == OK
        _check_select(s, q, out, K, 1, 2, lambda b: q)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e30, 3e38])
def test_queries_of_extreme_size(scale):
    s = Scored([6400], 2, 128, 64)
    q = (torch.randn(2, 4, 128, generator=s.c.g, device="cuda").clamp(-1, 1) * scale).to(BF)
    out, st = _select(s, q, 9, q_start=np.array([0, 2]))
    assert st == OK
    _check_select(s, q, out, 9, 1, 2, lambda b: q)


def test_selection_refusals_on_the_device():
    s = Scored([6400, 3000, 9000], 2, 64, 64)
    start, q = _chunks([2, 3, 1], 4, 64, s.c.g)
    rows = lambda b: q[start[b]:start[b + 1]]
    keep = s.c.d_ctx.clone()
    for bad, why in ((-1, INVALID), (16 * s.c.bt.shape[1] + 1, FULL), ((1 << 31) - 1, FULL)):
        s.c.d_ctx.copy_(keep)
        s.c.d_ctx[1] = bad
        out, st = _select(s, q, 9, q_start=start)
        assert st == why
        _check_select(s, q, out, 9, 1, 2, rows, skip=(1,))
    s.c.d_ctx.copy_(keep)
    for wrong in ([0, 2, 1, 6], [0, 2, 5, 7], [-1, 2, 5, 6]):
        bad = [b for b in range(3) if wrong[b] < 0 or wrong[b + 1] < wrong[b] or wrong[b + 1] > 6]
        out, st = _select(s, q, 9, q_start=np.array(wrong))
        assert st == INVALID
        _check_select(s, q, out, 9, 1, 2, lambda b: q[max(wrong[b], 0):wrong[b + 1]], skip=bad)
    for n in (-1, 2):
        out, st = _select(s, q[:3, None].contiguous(), 9, n=np.array([1, n, 1]))
        assert st == INVALID
        _check_select(s, q, out, 9, 1, 2, lambda b: q[b:b + 1], skip=(1,))
    at = int(s.c.bt[2, 12])                                                  # the first page of block 3
    s.c.block_table[2, 12] = s.c.num_pages
    s.scale[at] = 0
    out, st = _select(s, q, 9, q_start=start)
    assert st == INVALID
    _check_select(s, q, out, 9, 1, 2, rows)


def test_selection_of_no_rows_at_all():
    s = Scored([6400, 100], 2, 64, 64)
    out, st = _select(s, torch.empty(0, 4, 64, device="cuda", dtype=BF), 5, q_start=np.zeros(3, int))
    assert st == OK and (out == -1).all()


@pytest.mark.parametrize("n", [1, 9])
def test_many_rows_of_many_blocks(n):
    """Enough choices that a query rounded the other way anywhere, or a score off by one, changes some of them: 512 lists of 32 out of 512 blocks, by 4 queries (in registers) and
    by 36 (through shared memory)."""
    s = Scored([32768 - 17 * b for b in range(64)], 8, 128, 64, seed=n)
    start, q = _chunks([n] * 64, 32, 128, s.c.g)
    out, st = _select(s, q, 32, q_start=start, hints=True)
    assert st == OK
    rows = q.view(64, n, 8, 4, 128).permute(0, 2, 1, 3, 4).reshape(64, 8, n * 4, 128).float()
    top = rows.abs().amax((2, 3), keepdim=True)
    eighth = torch.round(rows * (torch.full_like(top, 127.0) / top)).to(F8)
    for b in range(64):
        at = s.first_pages(b)
        dot = torch.matmul(eighth[b], s.mean[at].to(F8).permute(1, 2, 0)).amax(1)            # [heads, blocks]
        score = dot.float() * s.scale[at].t()
        score[:, 0] = score[:, -2:] = math.inf
        best = torch.sort(score, dim=1, descending=True, stable=True)[1][:, :32].sort(1)[0]
        assert out[b].tolist() == best.tolist(), b
