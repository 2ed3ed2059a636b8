"""Which pages of a KV4Cache belong to which sequence: host-side bookkeeping, no GPU work.

A pool hands out pages, counts who holds them, and says which pages have to be copied (kv4_copy_pages) when a sequence is forked or
the pool is compacted.  It keeps Python integers; the caller uploads tables and copies when a step is launched."""
from __future__ import annotations

from typing import Dict, List, Tuple


class PagePool:
    """Pages 0 .. pages - 1 of page_size tokens.  Sequences are named by the caller."""

    def __init__(self, pages: int, page_size: int):
        if pages < 0 or page_size < 1:
            raise ValueError("pages must be >= 0 and page_size >= 1")
        self.page_size = int(page_size)
        self._free = list(range(int(pages) - 1, -1, -1))     # lowest numbers are handed out first
        self._held = [0] * int(pages)                        # sequences that hold a page
        self._tables: Dict[object, List[int]] = {}
        self._lens: Dict[object, int] = {}

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, seq) -> int:
        return self._lens[seq]

    def table(self, seq) -> List[int]:
        """The sequence's page numbers in order (a copy)."""
        return list(self._tables[seq])

    def _take(self) -> int:
        page = self._free.pop()
        self._held[page] = 1
        return page

    def _drop(self, page: int) -> None:
        self._held[page] -= 1
        if self._held[page] == 0:
            self._free.append(page)

    def add(self, seq) -> None:
        """A new, empty sequence."""
        if seq in self._tables:
            raise ValueError(f"sequence {seq!r} is there already")
        self._tables[seq], self._lens[seq] = [], 0

    def extend(self, seq, tokens: int) -> Tuple[List[int], List[Tuple[int, int]]]:
        """Room for `tokens` more tokens: (their slots, pages to copy first).  A page that other sequences hold too is copied
        before it is written to: (src, dst) pairs for kv4_copy_pages.  Pairs of consecutive calls of extend may be joined in one
        copy; they have to be launched before any other call that changes the pool (fork, truncate, free, compact): pages could be
        handed out again that are still to be read.  MemoryError where the pool has too few pages; nothing has changed then."""
        if tokens < 0:
            raise ValueError("tokens must be >= 0")
        if tokens == 0:
            return [], []
        p, table, n = self.page_size, self._tables[seq], self._lens[seq]
        shared = n % p != 0 and self._held[table[n // p]] > 1
        need = -(-(n + tokens) // p) - len(table) + shared
        if need > len(self._free):
            raise MemoryError(f"{need} pages are needed, {len(self._free)} are free")
        copies = []
        if shared:
            old, new = table[n // p], self._take()
            self._held[old] -= 1
            table[n // p] = new
            copies.append((old, new))
        while len(table) * p < n + tokens:
            table.append(self._take())
        self._lens[seq] = n + tokens
        return [table[i // p] * p + i % p for i in range(n, n + tokens)], copies

    def fork(self, seq, new) -> None:
        """A new sequence with all of seq's tokens.  It shares the pages; a partly filled one is copied when either writes to it."""
        if new in self._tables:
            raise ValueError(f"sequence {new!r} is there already")
        for page in self._tables[seq]:
            self._held[page] += 1
        self._tables[new], self._lens[new] = list(self._tables[seq]), self._lens[seq]

    def common_pages(self, seqs) -> int:
        """How many pages the sequences begin with in common, filled in all of them: kv4_prefix_attention reads these once.  Their numbers are
        the first ones of any of the tables; what is behind them is each sequence's own."""
        seqs = list(seqs)
        if not seqs:
            return 0
        n = min(self._lens[seq] for seq in seqs) // self.page_size
        first = self._tables[seqs[0]]
        for seq in seqs[1:]:
            table = self._tables[seq]
            n = next((i for i in range(n) if table[i] != first[i]), n)
        return n

    def shared_pages(self, seq) -> int:
        """How many of the sequence's pages other sequences hold too.  A sequence that has some is not evicted in place (kv4_evict without
        new_table): the others' tokens lie in the same pages."""
        return sum(self._held[page] > 1 for page in self._tables[seq])

    def truncate(self, seq, length: int) -> None:
        """The sequence's first `length` tokens; pages behind them are freed."""
        if not 0 <= length <= self._lens[seq]:
            raise ValueError("length must be in 0 .. the sequence's")
        table = self._tables[seq]
        while len(table) > -(-length // self.page_size):
            self._drop(table.pop())
        self._lens[seq] = length

    def free(self, seq) -> None:
        """The sequence is done; pages that nobody else holds are free again."""
        for page in self._tables.pop(seq):
            self._drop(page)
        del self._lens[seq]

    def compact(self) -> List[Tuple[int, int]]:
        """Moves held pages into the lowest free ones, so that the held pages are 0 .. held - 1: (src, dst) pairs for
        kv4_copy_pages, none of them both read and written.  The tables name the new pages when this returns: launch the copy
        before the next call that reads the cache."""
        held = [i for i, n in enumerate(self._held) if n]
        holes = [i for i in range(len(held)) if self._held[i] == 0]
        moved = dict(zip([i for i in held if i >= len(held)], holes))
        for src, dst in moved.items():
            self._held[dst], self._held[src] = self._held[src], 0
        for table in self._tables.values():
            table[:] = [moved.get(page, page) for page in table]
        self._free = list(range(len(self._held) - 1, len(held) - 1, -1))
        return list(moved.items())
