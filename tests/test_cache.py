"""Pages and rotation tables on the host."""
import numpy as np
import pytest

from paper_2607_16673_amd.cache import PagePool, rope_table


def check(pool, seqs):
    """Every page is free or held by as many sequences as list it."""
    count = np.zeros(len(pool.holders), int)
    for s in seqs:
        assert len(s.pages) == len(set(s.pages)) and len(s.pages) * pool.page_size >= s.length
        for p in s.pages:
            count[p] += 1
    assert count.tolist() == pool.holders
    assert sorted(pool._free) == np.flatnonzero(count == 0).tolist()


def test_reserve_and_free():
    pool = PagePool(5, 16)
    a = pool.new()
    assert pool.reserve(a, 0) == [] and a.pages == []
    assert pool.reserve(a, 1) == [] and len(a.pages) == 1
    assert pool.reserve(a, 16) == [] and len(a.pages) == 1
    a.length = 16
    assert pool.reserve(a, 16) == [] and len(a.pages) == 2
    a.length = 20
    assert pool.reserve(a, 13) == [] and len(a.pages) == 3
    b = pool.new()
    with pytest.raises(MemoryError):
        pool.reserve(b, 33)
    check(pool, [a, b])
    pool.reserve(b, 32)
    assert pool.free_pages == 0
    pool.free(a)
    check(pool, [a, b])
    assert pool.free_pages == 3 and a.length == 0


def test_fork_copies_what_is_written():
    pool = PagePool(10, 16)
    a = pool.new()
    pool.reserve(a, 50)
    a.length = 40  # two full pages, one of 8 rows, one reserved only
    b, c = pool.fork(a), pool.fork(a)
    assert b.pages == c.pages == a.pages[:3] and pool.free_pages == 6
    old = a.pages[2]
    assert pool.reserve(b, 0) == []
    assert pool.reserve(b, 4) == [(old, b.pages[2], 8)]
    assert pool.reserve(a, 20) == [(old, a.pages[2], 8)]
    assert pool.reserve(c, 20) == [] and c.pages[2] == old  # the last holder writes in place
    check(pool, [a, b, c])
    assert pool.reserve(b, 4) == []
    pool.free(a), pool.free(c)
    check(pool, [a, b, c])


def test_fork_at_a_page_boundary_and_truncation():
    pool = PagePool(10, 16)
    a = pool.new()
    pool.reserve(a, 48)
    a.length = 32
    b = pool.fork(a)
    assert len(b.pages) == 2 and pool.reserve(b, 1) == [] and b.pages[2] != a.pages[2]
    b.length = 33
    shared = a.pages[0], a.pages[1]
    pool.truncate(b, 5)
    assert b.pages == [shared[0]]
    assert pool.reserve(b, 20) == [(shared[0], b.pages[0], 5)]
    b.length = 16
    pool.truncate(a, 0)
    check(pool, [a, b])
    assert a.pages == []
    for bad in (17, -1):
        with pytest.raises(ValueError):
            pool.truncate(b, bad)


def test_whole_pages_that_are_written_again_are_not_copied():
    pool = PagePool(6, 16)
    a = pool.new()
    pool.reserve(a, 32)
    a.length = 32
    b = pool.fork(a)
    pool.truncate(b, 16)
    assert len(b.pages) == 1
    b.pages.append(a.pages[1])  # as a caller that keeps the page might hold it
    pool.holders[a.pages[1]] += 1
    assert pool.reserve(b, 16) == [] and b.pages[1] != a.pages[1]
    check(pool, [a, b])


def test_memory_errors_change_nothing():
    pool = PagePool(4, 16)
    a = pool.new()
    pool.reserve(a, 40)
    a.length = 40
    b = pool.fork(a)
    before = list(b.pages), list(pool.holders), list(pool._free)
    with pytest.raises(MemoryError):
        pool.reserve(b, 30)
    assert before == (b.pages, pool.holders, pool._free)
    pool.reserve(b, 8)
    check(pool, [a, b])


def test_random_lives():
    rng = np.random.default_rng(0)
    pool, seqs = PagePool(64, 16), []
    for _ in range(2000):
        what = rng.integers(5)
        if what == 0 or not seqs:
            seqs.append(pool.new())
        s = seqs[rng.integers(len(seqs))]
        if what == 1:
            seqs.append(pool.fork(s))
        elif what == 2:
            pool.truncate(s, int(rng.integers(s.length + 1)))
        elif what == 3 and len(seqs) > 3:
            pool.free(s)
            seqs.remove(s)
        else:
            n = int(rng.integers(1, 64))
            try:
                copies = pool.reserve(s, n)
            except MemoryError:
                pool.free(s)
                continue
            assert all(pool.holders[dst] == 1 and pool.holders[src] >= 1 and 0 < rows < 16 for src, dst, rows in copies)
            assert all(pool.holders[p] == 1 for p in s.pages[s.length // 16:-(-(s.length + n) // 16)])
            s.length += int(rng.integers(n + 1))
        check(pool, seqs)


def test_table():
    pool = PagePool(9, 32)
    a, b = pool.new(), pool.new()
    pool.reserve(a, 70), pool.reserve(b, 5)
    t = pool.table([b, a])
    assert t.dtype == np.int32 and t.tolist() == [b.pages + [-1, -1], a.pages]
    assert pool.table([b], 4).shape == (1, 4) and pool.table([pool.new()]).tolist() == [[-1]]


def test_refusals():
    for pages, size in ((0, 16), (4, 8), (4, 24), (4, 512)):
        with pytest.raises(ValueError):
            PagePool(pages, size)
    with pytest.raises(ValueError):
        PagePool(4, 16).reserve(PagePool(4, 16).new(), -1)
    for bad in (dict(length=0, dim=8), dict(length=4, dim=7), dict(length=4, dim=0), dict(length=4, dim=8, factor=0.0),
                dict(length=4, dim=8, frequencies=[1.0] * 8)):
        with pytest.raises(ValueError):
            rope_table(**bad, device="cpu")


def test_rope_table():
    pos, i = np.arange(300000)[:, None], np.arange(8)
    for kw, f, factor in [({}, 1e4 ** (-i / 8), 1.0), (dict(base=5e5, factor=4.0), 5e5 ** (-i / 8), 4.0),
                          (dict(frequencies=1.0 / (i + 1)), 1.0 / (i + 1), 1.0)]:
        t = rope_table(300000, 16, device="cpu", **kw).numpy()
        angle = pos / factor * f
        assert t.dtype == np.float32 and t.shape == (300000, 16)
        # rounded once: half a unit in the last place of 1, and the angle's 2^-53 of 3e5
        assert np.abs(t - np.concatenate([np.cos(angle), np.sin(angle)], 1)).max() <= 2.0 ** -25 + 2.0 ** -30
