"""cb_pages_assign and cb_slot_map against plain loops: every page, count and slot equal."""
import numpy as np
import pytest
import torch

from tests.block_refs import assign
from tests.operator_refs import PAGE, Paged, context, cuda

pytestmark = pytest.mark.gpu
OK, INVALID, FULL = 0, 1, 8


class Pool:
    def __init__(self, held, width, spare, seed=0):
        rng = np.random.default_rng(seed)
        self.held = np.asarray(held, np.int64)
        total = int(self.held.sum()) + spare
        ids = rng.permutation(total)
        self.table = rng.integers(-9, -1, (len(held), width))
        at = 0
        for b, k in enumerate(held):
            self.table[b, :k] = ids[at:at + k]
            at += k
        self.free = np.full(max(total, 1), -7, np.int64)
        self.free[:spare] = ids[at:]
        self.n_free = spare
        self.d = [cuda(x) for x in (self.table, self.held, self.free, np.array([spare]))]
        self.cb = context(batch=len(held))

    def call(self, want):
        t, h, f, n = self.d
        self.cb.cb_pages_assign(cuda(np.asarray(want)), t, h, f, n)
        return self.cb.cb_poll_status()[0]

    def step(self, want):
        st = self.call(want)
        self.n_free, alone = assign(want, self.table, self.held, self.free, self.n_free)
        assert st == (FULL if alone else OK)
        self.check()

    def check(self):
        for got, ref in zip(self.d, (self.table, self.held, self.free, np.array([self.n_free]))):
            assert np.array_equal(got.cpu().numpy(), ref)


@pytest.mark.parametrize("batch,width,spare,top", [(1, 1, 1, 16), (1, 40, 20, 600), (3, 9, 10, 140), (32, 33, 400, 512), (31, 700, 9000, 9000),
                                                   (1000, 12, 3000, 190), (1025, 20, 9000, 300), (2500, 8, 9000, 120), (513, 600, 150000, 8192)])
def test_random_steps(batch, width, spare, top):
    rng = np.random.default_rng(batch + width)
    p = Pool(np.zeros(batch, int), width, spare)
    for step in range(6):
        want = rng.integers(0, top + 1, batch)
        if step == 3:
            want = np.where(rng.random(batch) < 0.5, 0, p.held * PAGE)      # some finish, nobody grows
        p.step(want)


def test_a_step_taken_back_leaves_the_stack_as_it_was():
    rng = np.random.default_rng(1)
    p = Pool(rng.integers(0, 20, 50), 64, 2000)
    free, n = p.free.copy(), p.n_free
    back = p.held * PAGE
    p.step(back + rng.integers(0, 300, 50))
    assert p.n_free < n
    p.step(back)
    assert p.n_free == n and np.array_equal(p.free, free)


def test_pages_given_back_go_to_those_that_grow_in_the_same_call():
    p = Pool([4, 0, 3, 1], 8, 0)
    mine = p.table[0, 1:4].tolist() + p.table[2, :3].tolist()
    p.step([16, 40, 0, 30])
    assert p.table[1, :3].tolist() + p.table[3, 1:2].tolist() == mine[:4] and p.n_free == 2


@pytest.mark.parametrize("spare,ok", [(5, [True, True, True]), (4, [True, True, False]), (3, [True, False, False]), (1, [True, False, False]), (0, [False] * 3)])
def test_too_few_pages(spare, ok):
    """In order of the batch; behind one that does not fit nobody grows, but pages are still given back."""
    p = Pool([1, 0, 2, 1], 8, spare)
    p.step([32, 16 * 3, 32, 17])
    assert (p.held == [1 + ok[0], 3 * ok[1], 2, 1 + ok[2]]).all()
    p.step([0, 0, 0, 0])
    assert p.n_free == spare + 4


def test_what_is_left_alone():
    p = Pool([2, 3, 1, 0], 4, 6)
    assert p.call([16, 65, 16, 16]) == FULL                                  # five pages in a table of four
    p.n_free, _ = assign([16, 65, 16, 16], p.table, p.held, p.free, p.n_free)
    p.check()
    assert p.call([16, -1, 16, 16]) == INVALID                               # keeps its three pages
    p.check()
    for bad in (-1, 5, 1 << 30):
        p.d[1][1] = bad
        assert p.call([16, 0, 16, 16]) == INVALID
        assert int(p.d[1][1]) == bad
    p.d[1][1] = 3
    p.check()
    for bad in (-1, 13, 1 << 30, -(1 << 31)):
        p.d[3][0] = bad
        assert p.call([64, 64, 0, 0]) == INVALID
        p.d[3][0] = p.n_free
        p.check()
    p.d[3][0] = 12                                                           # pages given back would not fit the stack
    assert p.call([0, 0, 0, 0]) == INVALID
    p.d[3][0] = p.n_free
    p.check()


def test_growth_by_pages_and_length_borders():
    p = Pool([0], 300, 299)
    for want in (1, 15, 16, 17, 32, 33, 4784, 0, 4784, 4783, 4769, 4768):
        p.step([want])


def _map(c, n_rows, width=None):
    cb = context(batch=len(c.new))
    new = lambda t: torch.full((n_rows,), 77, device="cuda", dtype=t)
    res = dict(slots=new(torch.int64), positions=new(torch.int32), seqs=new(torch.int32))
    cb.cb_slot_map(c.d_start, c.d_ctx, c.block_table, c.num_pages, n_rows, res=res)
    return {k: v.cpu().numpy() for k, v in res.items()}, cb.cb_poll_status()[0]


def _expect(c, n_rows, skip=()):
    ref = {k: np.full(n_rows, -1, np.int64) for k in ("slots", "positions", "seqs")}
    for b in range(len(c.new)):
        if b in skip:
            continue
        pos = c.ctx[b] + np.arange(c.new[b])
        rows = np.arange(c.q_start[b], c.q_start[b + 1])
        ref["slots"][rows], ref["positions"][rows], ref["seqs"][rows] = c.bt[b, pos // PAGE] * PAGE + pos % PAGE, pos, b
    return ref


@pytest.mark.parametrize("new,ctx,pad", [([1], [0], 0), ([0], [5], 3), ([1] * 32, list(range(100, 132)), 0), ([0, 300, 0, 0, 17, 1, 0], [9, 0, 3, 1, 16, 31, 2], 5),
                                         ([256], [15], 0), ([257, 1], [16, 255], 512), ([5000, 3], [0, 4000], 1)])
def test_slots(new, ctx, pad):
    c = Paged(new, ctx, 1, 64, seed=3)
    n = int(c.q_start[-1]) + pad
    got, st = _map(c, n)
    ref = _expect(c, n)
    assert st == OK
    for k in ref:
        assert np.array_equal(got[k], ref[k]), k


@pytest.mark.parametrize("batch", [2047, 2048, 2049, 5000])
def test_slots_of_many_sequences(batch):
    rng = np.random.default_rng(batch)
    c = Paged(rng.integers(0, 4, batch), rng.integers(0, 60, batch), 1, 64)
    n = int(c.q_start[-1]) + 7
    got, st = _map(c, n)
    ref = _expect(c, n)
    assert st == OK and all(np.array_equal(got[k], ref[k]) for k in ref)


def test_slots_beyond_32_bits():
    c = Paged([3], [14], 1, 64)
    big = (1 << 31) - 2
    c.bt[0, :2] = big - 5, big
    c.block_table, c.num_pages = cuda(c.bt), (1 << 31) - 1
    got, st = _map(c, 3)
    assert st == OK and got["slots"].tolist() == [(big - 5) * 16 + 14, (big - 5) * 16 + 15, big * 16]


def test_rows_before_the_first_sequence_and_bad_sequences():
    c = Paged([3, 4, 5, 2], [10, 20, 30, 40], 1, 64)
    c.q_start = c.q_start + 2
    c.d_start = cuda(c.q_start)
    n = 20
    got, st = _map(c, n)
    ref = _expect(c, n)
    assert st == OK and all(np.array_equal(got[k], ref[k]) for k in ref) and got["seqs"][:2].tolist() == [-1, -1]
    for ctx, why in ((-1, INVALID), (16 * c.bt.shape[1] - 3, FULL), ((1 << 31) - 1, FULL), (-(1 << 31), INVALID)):
        c.d_ctx = cuda(c.ctx)
        c.d_ctx[1] = ctx
        got, st = _map(c, n)
        ref = _expect(c, n, skip=(1,))
        assert st == why and all(np.array_equal(got[k], ref[k]) for k in ref), ctx
    c.d_ctx = cuda(c.ctx)
    got, st = _map(c, 15)                                                    # the last sequence's range ends behind the rows
    ref = _expect(c, 20, skip=(3,))
    assert st == INVALID and all(np.array_equal(got[k], ref[k][:15]) for k in ref)
    c.block_table[2, 2] = c.num_pages                                        # a page outside the pool
    got, st = _map(c, n)
    ref = _expect(c, n)
    at = np.nonzero((ref["seqs"] == 2) & (ref["positions"] // 16 == 2))[0]
    assert len(at) and st == INVALID
    ref["slots"][at] = -1
    assert all(np.array_equal(got[k], ref[k]) for k in ref)
