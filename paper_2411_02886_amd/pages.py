"""Which pages of a paged KV pool belong to which sequence: taking, sharing, copying on write, moving together and giving back.

The table lives on the host, where a server decides what runs next; the pages' contents are moved by ts_pages_copy, once per
layer, with the (source, destination) lists that the methods here return, one after the other (copy_runs).  Nothing here touches a page.
"""
from __future__ import annotations

import heapq

import numpy as np


def copy_runs(copies):
    """The list [(src, dst)] cut into runs [(begin, end)] whose copies need no order among them, as ts_pages_copy wants them: no page of a
    run is written twice, or written by one pair and read by another."""
    runs, begin, read, written = [], 0, set(), set()
    for i, (a, b) in enumerate(copies):
        if a == b:
            continue
        if a in written or b in written or b in read:
            runs.append((begin, i))
            begin, read, written = i, set(), set()
        read.add(a)
        written.add(b)
    if len(copies) > begin:
        runs.append((begin, len(copies)))
    return runs


class PagePool:
    """Pages 0 .. num_pages - 1 of `page_size` tokens.  A page may belong to several sequences (fork); the lowest free page is
    taken first, so that a pool that empties stays dense at its low end.  Sequences go by any hashable name.  A call that
    cannot be served raises and changes nothing."""

    def __init__(self, num_pages: int, page_size: int):
        if num_pages < 1 or page_size < 1:
            raise ValueError("a pool has at least one page of at least one token")
        self.num_pages, self.page_size = int(num_pages), int(page_size)
        self.refs = np.zeros(self.num_pages, dtype=np.int32)      # sequences that hold the page
        self._free = list(range(self.num_pages))                  # a heap
        self._pages, self._lens, self._spare = {}, {}, set()

    def __contains__(self, seq):
        return seq in self._pages

    def __len__(self):
        return len(self._pages)

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, seq) -> int:
        return self._lens[seq]

    def pages(self, seq):
        return list(self._pages[seq])

    def _take(self, n: int):
        got = [heapq.heappop(self._free) for _ in range(n)]
        self.refs[got] += 1
        return got

    def _release(self, pages):
        for page in pages:
            self.refs[page] -= 1
            if self.refs[page] == 0:
                heapq.heappush(self._free, page)

    def add(self, seq, tokens: int = 0) -> None:
        """A new sequence of `tokens` tokens."""
        if seq in self._pages:
            raise KeyError("sequence %r is there already" % (seq,))
        if tokens < 0:
            raise ValueError("tokens < 0")
        need = -(-tokens // self.page_size)
        if need > len(self._free):
            raise MemoryError("%d pages wanted, %d free" % (need, len(self._free)))
        self._pages[seq], self._lens[seq] = self._take(need), int(tokens)

    def grow(self, seq, tokens: int = 1):
        """Room for `tokens` more tokens.  Returns the page copies, [(src, dst)], to be made before the new tokens are written: a
        last page that is partly filled and shared is replaced by a copy of its own."""
        if tokens < 0:
            raise ValueError("tokens < 0")
        pages, n = self._pages[seq], self._lens[seq]
        need = -(-(n + tokens) // self.page_size) - len(pages)
        own = tokens > 0 and n % self.page_size != 0 and self.refs[pages[-1]] > 1
        if need + own > len(self._free):
            raise MemoryError("%d pages wanted, %d free" % (need + own, len(self._free)))
        copies = []
        if own:
            page = self._take(1)[0]
            copies.append((pages[-1], page))
            self.refs[pages[-1]] -= 1           # another sequence holds it: it does not become free
            pages[-1] = page
        pages += self._take(max(need, 0))
        self._lens[seq] = n + int(tokens)
        return copies

    def fork(self, seq, child) -> None:
        """`child` begins as `seq` is now and shares its pages."""
        if child in self._pages:
            raise KeyError("sequence %r is there already" % (child,))
        pages = self._pages[seq]
        self.refs[pages] += 1
        self._pages[child], self._lens[child] = list(pages), self._lens[seq]

    def free(self, seq) -> None:
        """Gives the sequence's pages back; those that another one holds stay."""
        self._release(self._pages.pop(seq))
        del self._lens[seq]

    def spare(self, tokens: int):
        """Pages for `tokens` tokens that belong to no sequence yet: where a compaction writes (see replace, give_back)."""
        if tokens < 0:
            raise ValueError("tokens < 0")
        need = -(-int(tokens) // self.page_size)
        if need > len(self._free):
            raise MemoryError("%d pages wanted, %d free" % (need, len(self._free)))
        pages = self._take(need)
        self._spare.update(pages)
        return pages

    def _of_spare(self, pages):
        pages = [int(page) for page in pages]
        if len(set(pages)) != len(pages) or not self._spare.issuperset(pages):
            raise ValueError("pages that are not spare, or one of them twice")
        return pages

    def give_back(self, pages) -> None:
        """Returns spare pages that were not used."""
        pages = self._of_spare(pages)
        self._spare.difference_update(pages)
        self._release(pages)

    def replace(self, seq, pages, tokens: int) -> None:
        """The sequence now is the first `tokens` tokens of the spare `pages` (what a compaction wrote); its old pages and
        those that the tokens do not reach are given back."""
        need = -(-int(tokens) // self.page_size)
        if tokens < 0 or need > len(pages):
            raise ValueError("%d tokens do not fit %d pages" % (tokens, len(pages)))
        old, pages = self._pages[seq], self._of_spare(pages)
        self._spare.difference_update(pages)
        self._pages[seq], self._lens[seq] = list(pages[:need]), int(tokens)
        self._release(old)
        self._release(pages[need:])

    def gather(self):
        """Moves the sequences' pages to the low end of the pool, the highest to the lowest free place; spare pages, which the caller
        goes by, stay.  Returns the page copies, [(src, dst)], to be made before the next page is written; no page is in both columns."""
        high = [int(page) for page in np.flatnonzero(self.refs)[::-1] if int(page) not in self._spare]
        moved = [(a, b) for a, b in zip(high, sorted(self._free)) if a > b]
        to = dict(moved)
        for pages in self._pages.values():
            pages[:] = [to.get(page, page) for page in pages]
        for a, b in moved:
            self.refs[b], self.refs[a] = self.refs[a], 0
        self._free = [int(page) for page in np.flatnonzero(self.refs == 0)]     # ascending: a heap
        return moved

    def table(self, seqs, room: int = 0):
        """(page_indptr [B+1], page_indices, seq_lens [B]) of the sequences, int32, as ts_problem wants them.  room: empty
        places in page_indices behind each sequence's pages, for pages it will get."""
        rows = [self._pages[s] + [0] * room for s in seqs]
        indptr = np.cumsum([0] + [len(r) for r in rows], dtype=np.int64)
        if indptr[-1] > np.iinfo(np.int32).max:
            raise ValueError("more pages than an int32 counts")
        return (indptr.astype(np.int32), np.array([page for r in rows for page in r] or [0], dtype=np.int32),
                np.array([self._lens[s] for s in seqs], dtype=np.int32))
