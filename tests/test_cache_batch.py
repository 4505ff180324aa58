"""Reservations for a whole batch: all of it or nothing."""
import copy

import numpy as np
import pytest

from paper_2607_16673_amd.cache import PagePool
from test_cache import check


def shared(pool, rows, count):
    """A sequence of `rows` rows and its forks."""
    a = pool.new()
    pool.reserve(a, rows)
    a.length = rows
    return [a] + [pool.fork(a) for _ in range(count - 1)]


def state(pool, seqs):
    return copy.deepcopy(([(s.length, s.pages) for s in seqs], pool.holders, pool._free))


def test_too_few_pages_for_the_last_sequence_change_nothing():
    """Three sequences that share a half page, one page free: the first would get
    it, the second has none; a later try still copies the rows of the first."""
    pool = PagePool(4, 16)
    seqs = shared(pool, 40, 3)
    old = seqs[0].pages[2]
    before = state(pool, seqs)
    with pytest.raises(MemoryError):
        pool.reserve_all(seqs, 4)
    assert state(pool, seqs) == before
    pool.free(seqs.pop())
    assert pool.reserve_all(seqs, 4) == [(old, seqs[0].pages[2], 8)]
    assert seqs[1].pages[2] == old
    check(pool, seqs)


def test_the_last_holder_keeps_its_page():
    """Two of three holders copy: two pages, not three, are enough."""
    pool = PagePool(5, 16)
    seqs = shared(pool, 40, 3)
    old = seqs[0].pages[2]
    copies = pool.reserve_all(seqs, 8)
    assert copies == [(old, seqs[0].pages[2], 8), (old, seqs[1].pages[2], 8)] and seqs[2].pages[2] == old
    assert pool.free_pages == 0
    check(pool, seqs)


def test_as_one_by_one():
    """With pages enough it does what a reservation of each in turn does."""
    rng = np.random.default_rng(0)
    for _ in range(300):
        pool = PagePool(200, 16)
        seqs = []
        for _ in range(int(rng.integers(1, 5))):
            seqs += shared(pool, int(rng.integers(0, 70)), int(rng.integers(1, 4)))
        for s in seqs:
            if rng.integers(3) == 0:
                pool.truncate(s, int(rng.integers(s.length + 1)))
        seqs = [seqs[i] for i in rng.permutation(len(seqs))]
        rows = int(rng.integers(0, 40))
        twin, twins = copy.deepcopy((pool, seqs))
        want = [c for s in twins for c in twin.reserve(s, rows)]
        used = pool.free_pages - twin.free_pages
        tight, ts = copy.deepcopy((pool, seqs))
        del tight._free[:len(tight._free) - used]  # just enough
        for p, q in ((pool, seqs), (tight, ts)):
            assert p.reserve_all(q, rows) == want and [s.pages for s in q] == [s.pages for s in twins]
            assert p.holders == twin.holders
        check(pool, seqs)
        assert tight.free_pages == 0 or used == 0
        dst = [d for _, d, _ in want]
        assert len(set(dst)) == len(dst) and not set(dst) & {s for s, _, _ in want}  # as sla_page_copy asks


def test_refusals():
    pool = PagePool(9, 16)
    a, b = pool.new(), pool.new()
    with pytest.raises(ValueError):
        pool.reserve_all([a, b], -1)
    with pytest.raises(ValueError):
        pool.reserve_all([a, b, a], 3)
    assert pool.reserve_all([], 5) == [] and pool.reserve_all([a, b], 0) == [] and pool.free_pages == 9
