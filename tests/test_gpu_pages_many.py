"""cb_pages_assign where a table is large enough for several CTAs (more than 65,536 entries): what is left alone, what is recorded, and that the next call finds
everything as it should be."""
import numpy as np
import pytest

from tests.block_refs import assign
from tests.test_gpu_pages import FULL, INVALID, Pool

pytestmark = pytest.mark.gpu
WIDE = 40000                                                                 # columns: with four sequences a CTA for every 2,048 entries, 78


def _good(p, want):
    """A call that has to succeed on the same context: a count of CTAs left over from the one before would leave held and n_free as they were."""
    p.step(want)
    assert (p.held == -(-np.asarray(want) // 16)).all()


@pytest.mark.parametrize("spare,ok", [(5, [True, True, True]), (4, [True, True, False]), (3, [True, False, False]), (1, [True, False, False]), (0, [False] * 3)])
def test_too_few_pages(spare, ok):
    p = Pool([1, 0, 2, 1], WIDE, spare)
    p.step([32, 16 * 3, 32, 17])
    assert (p.held == [1 + ok[0], 3 * ok[1], 2, 1 + ok[2]]).all()
    _good(p, [0, 0, 0, 0])
    assert p.n_free == spare + 4
    _good(p, [16, 0, 1, 32])


def test_what_is_left_alone():
    p = Pool([2, 3, 1, 0], WIDE, 6)
    over = 16 * WIDE + 1
    assert p.call([16, over, 16, 16]) == FULL                                # a page more than a table has
    p.n_free, _ = assign([16, over, 16, 16], p.table, p.held, p.free, p.n_free)
    p.check()
    _good(p, [32, 48, 16, 0])
    assert p.call([32, -1, 16, 16]) == INVALID                               # keeps its three pages
    p.n_free, _ = assign([32, 48, 16, 16], p.table, p.held, p.free, p.n_free)
    p.check()
    for bad in (-1, WIDE + 1, 1 << 30, -(1 << 31)):
        p.d[1][1] = bad
        assert p.call([32, 0, 16, 16]) == INVALID
        assert int(p.d[1][1]) == bad
        p.d[1][1] = 3
        p.check()
    _good(p, [0, 100, 16, 16])
    for bad in (-1, len(p.free) + 1, 1 << 30, -(1 << 31)):
        p.d[3][0] = bad
        assert p.call([64, 64, 0, 0]) == INVALID
        assert int(p.d[3][0]) == bad
        p.d[3][0] = p.n_free
        p.check()
    _good(p, [64, 48, 1, 0])
    p.d[3][0] = len(p.free)                                                  # pages given back would not fit the stack
    assert p.call([0, 0, 0, 0]) == INVALID
    p.d[3][0] = p.n_free
    p.check()
    _good(p, [0, 0, 0, 0])
    assert p.n_free == 12


def test_an_admission_that_runs_out_of_pages():
    """513 sequences that want 40,000 pages more than there are, while some finish; then all that fits."""
    rng = np.random.default_rng(3)
    p = Pool(rng.integers(0, 200, 513), 600, 30000)
    for _ in range(4):
        want = np.where(rng.random(513) < 0.3, 0, rng.integers(0, 600 * 16 + 1, 513))
        before = p.held.copy()
        p.step(want)
        goal = -(-want // 16)
        assert ((p.held == goal) | ((p.held == before) & (goal > before))).all() and (p.held < goal).any()
        _good(p, p.held * 16 - rng.integers(0, 16, 513) * (p.held > 0))
    _good(p, np.zeros(513, int))
