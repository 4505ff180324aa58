"""Host side of the paged cache: which pages hold which sequence, and the
rotation's table.

    pool = PagePool(n_pages, page_size)
    a = pool.new()
    copies = pool.reserve(a, n)     # room for n rows behind the committed ones
    ...                             # append, verify, commit with pool.table([a, ...])
    a.length += accepted
    b = pool.fork(a)                # shares a's pages until one of them writes
    copies = pool.reserve_all([a, b], n)  # [(src, dst, rows)] for sla_page_copy
    pool.free(a)

The pool only keeps numbers; the pages are the caller's tensors.
"""
from __future__ import annotations

import numpy as np


class Sequence:
    """A sequence's committed rows and its pages, in order."""

    def __init__(self):
        self.length = 0
        self.pages = []


class PagePool:
    """Pages of a cache, counted: a page belongs to all the sequences that
    forked while they had it, and is copied when one of them is about to write
    to it."""

    def __init__(self, n_pages: int, page_size: int):
        if n_pages < 1 or page_size not in (16, 32, 64, 128, 256):
            raise ValueError("a pool has at least one page of 16, 32, 64, 128 or 256 rows")
        self.page_size = page_size
        self.holders = [0] * n_pages
        self._free = list(range(n_pages - 1, -1, -1))

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def new(self) -> Sequence:
        return Sequence()

    def reserve(self, seq: Sequence, rows: int):
        """Give `seq` pages of its own for the rows length..length + rows - 1.
        Returns the copies [(src, dst, rows)] that have to be made, in all layers,
        before those rows are written and before a page is freed.  Raises
        MemoryError, with nothing changed, if there are too few pages."""
        return self.reserve_all([seq], rows)

    def reserve_all(self, seqs, rows: int):
        """`reserve` for every sequence of a batch, all or none of it: after a
        MemoryError no sequence has changed.  (Of several calls of `reserve` the
        copies of those before the error still have to be made.)"""
        if rows < 0:
            raise ValueError("rows must not be negative")
        if len(set(seqs)) < len(seqs):
            raise ValueError("a batch has each sequence once")
        if rows == 0:
            return []
        size = self.page_size
        need, plan, left = 0, [], {}  # left: how often the batch's earlier sequences leave a page for a copy
        for seq in seqs:
            first, end = seq.length // size, -(-(seq.length + rows) // size)
            shared = []
            for i in range(first, min(end, len(seq.pages))):
                p = seq.pages[i]
                if self.holders[p] - left.get(p, 0) > 1:
                    left[p] = left.get(p, 0) + 1
                    shared.append(i)
            need += len(shared) + max(end - len(seq.pages), 0)
            plan.append((seq, first, end, shared))
        if need > len(self._free):
            raise MemoryError("%d pages needed, %d free" % (need, len(self._free)))
        copies = []
        for seq, first, end, shared in plan:
            for i in shared:
                src, seq.pages[i] = seq.pages[i], self._take()
                self.holders[src] -= 1
                if i == first and seq.length % size:
                    copies.append((src, seq.pages[i], seq.length % size))
            while len(seq.pages) < end:
                seq.pages.append(self._take())
        return copies

    def fork(self, seq: Sequence) -> Sequence:
        """A sequence with the same committed rows, in the same pages."""
        child = Sequence()
        child.length = seq.length
        child.pages = seq.pages[:-(-seq.length // self.page_size)]
        for p in child.pages:
            self.holders[p] += 1
        return child

    def truncate(self, seq: Sequence, length: int):
        """Forget the rows from `length` on and give back the pages behind them."""
        if not 0 <= length <= seq.length:
            raise ValueError("a sequence of %d rows has no prefix of %d" % (seq.length, length))
        keep = -(-length // self.page_size)
        self._drop(seq.pages[keep:])
        del seq.pages[keep:]
        seq.length = length

    def free(self, seq: Sequence):
        """Give back all of a sequence's pages."""
        self._drop(seq.pages)
        seq.pages, seq.length = [], 0

    def table(self, seqs, width: int = 0) -> np.ndarray:
        """The page table [len(seqs)][width] int32 (width 0: the longest's),
        -1 past a sequence's last page."""
        width = max([width, 1] + [len(s.pages) for s in seqs])
        out = np.full((len(seqs), width), -1, np.int32)
        for row, s in zip(out, seqs):
            row[:len(s.pages)] = s.pages
        return out

    def _take(self) -> int:
        p = self._free.pop()
        self.holders[p] = 1
        return p

    def _drop(self, pages):
        for p in pages:
            self.holders[p] -= 1
            if self.holders[p] == 0:
                self._free.append(p)


def rope_table(length: int, dim: int, base: float = 1e4, *, factor: float = 1.0, frequencies=None, device="cuda"):
    """The rotation table [length][dim] fp32 of sla_attn_append: row p holds
    cos and then sin of p / factor times the dim / 2 frequencies, which are
    base^(-2 i / dim) unless given.  Angles are taken in 64 bits: in 32, a
    position of 10^5 would be off by up to 2^-8.  Longer contexts than a model
    learned are a factor or frequencies of their own."""
    import torch

    if length < 1 or dim < 2 or dim % 2 or not factor > 0:
        raise ValueError("a table has at least one position, an even number of elements and a positive factor")
    if frequencies is None:
        f = base ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=device) / dim)
    else:
        f = torch.as_tensor(frequencies, dtype=torch.float64, device=device)
        if f.shape != (dim // 2,):
            raise ValueError("%d elements turn by %d frequencies, got %s" % (dim, dim // 2, tuple(f.shape)))
    angle = (torch.arange(length, dtype=torch.float64, device=device) / factor)[:, None] * f
    return torch.cat([angle.cos(), angle.sin()], 1).float()
