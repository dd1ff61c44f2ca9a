"""Which pages of a key/value cache belong to which sequence: the bookkeeping, on the host, of what `binding.attn_paged_append`, `attn_paged_fwd` and
`attn_paged_copy` work on.

Sequences may share pages: `fork` makes a second sequence of the same tokens that copies nothing, and a shared page is copied when one of the two is about
to write into it.  `extend` and `compact` return the copies that the caches need, as (source, destination) pairs for `attn_paged_copy`; they have to
be made, in the order of the calls, before the caches are used again.
"""
from __future__ import annotations

import heapq
from typing import List, Sequence, Tuple

import torch

Pairs = List[Tuple[int, int]]


class OutOfPages(RuntimeError):
    """There are fewer free pages than a call needs; it has changed nothing."""


class PageTable:
    """Pages 0 .. pages - 1 of `page_size` tokens each, dealt out to sequences, lowest number first."""

    def __init__(self, pages: int, page_size: int):
        if pages < 1:
            raise ValueError("a cache has at least one page")
        if page_size < 16 or page_size > 4096 or page_size & (page_size - 1):
            raise ValueError("page_size must be a power of two from 16 to 4096")
        self.pages, self.page_size = pages, page_size
        self._free = list(range(pages))      # a heap
        self._users = [0] * pages            # sequences that hold a page
        self._held = {}                      # sequence -> its pages in order
        self._length = {}
        self._next = 0

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, seq: int) -> int:
        return self._length[seq]

    def pages_of(self, seq: int) -> List[int]:
        return list(self._held[seq])

    def _new(self, held: List[int], length: int) -> int:
        seq, self._next = self._next, self._next + 1
        self._held[seq], self._length[seq] = held, length
        return seq

    def add(self) -> int:
        """A new, empty sequence."""
        return self._new([], 0)

    def fork(self, seq: int) -> int:
        """A new sequence of the same tokens, on the same pages."""
        held = list(self._held[seq])
        for p in held:
            self._users[p] += 1
        return self._new(held, self._length[seq])

    def free(self, seq: int) -> None:
        """Ends a sequence; pages that no other one holds are free again."""
        for p in self._held.pop(seq):
            self._users[p] -= 1
            if self._users[p] == 0:
                heapq.heappush(self._free, p)
        del self._length[seq]

    def extend(self, seqs: Sequence[int], tokens: Sequence[int]) -> Pairs:
        """Makes room for `tokens[i]` more tokens of sequence seqs[i], which counts them as its own from here on, and returns the copies that the caches need
        before those are appended: of pages that are shared and about to be written.  Raises OutOfPages with nothing changed."""
        if len(seqs) != len(tokens) or len(set(seqs)) != len(seqs):
            raise ValueError("one number of tokens for each sequence, and every sequence once")
        if any(n < 0 for n in tokens):
            raise ValueError("numbers of tokens are not negative")
        plan, users = [], {}
        need = 0
        for seq, n in zip(seqs, tokens):
            held, length = self._held[seq], self._length[seq]
            shared = None
            if n > 0 and length % self.page_size:
                p = held[length // self.page_size]
                if users.get(p, self._users[p]) > 1:
                    shared = length // self.page_size
                    users[p] = users.get(p, self._users[p]) - 1     # the last one to write keeps the page
            more = max(0, -(-(length + n) // self.page_size) - len(held))
            plan.append((seq, n, shared, more))
            need += more + (shared is not None)
        if need > len(self._free):
            raise OutOfPages(f"{need} pages needed, {len(self._free)} free")
        copies: Pairs = []
        for seq, n, shared, more in plan:
            held = self._held[seq]
            if shared is not None:
                p = heapq.heappop(self._free)
                copies.append((held[shared], p))
                self._users[held[shared]] -= 1
                self._users[p] = 1
                held[shared] = p
            for _ in range(more):
                p = heapq.heappop(self._free)
                self._users[p] = 1
                held.append(p)
            self._length[seq] += n
        return copies

    def compact(self) -> Pairs:
        """Moves pages so that those in use are the lowest numbers; returns the copies that the caches need."""
        used = self.pages - len(self._free)
        moves = dict(zip((p for p in range(used, self.pages) if self._users[p]), sorted(p for p in self._free if p < used)))
        for held in self._held.values():
            held[:] = [moves.get(p, p) for p in held]
        for src, dst in moves.items():
            self._users[dst], self._users[src] = self._users[src], 0
        self._free = list(range(used, self.pages))
        return list(moves.items())

    def batch(self, seqs: Sequence[int], device="cuda") -> Tuple[torch.Tensor, torch.Tensor]:
        """(block_table, lengths) of these sequences, int32, as the calls take them; a row is filled up with -1, which is no page."""
        rows = [self._held[s] for s in seqs]
        width = max(1, max((len(r) for r in rows), default=1))
        table = torch.tensor([r + [-1] * (width - len(r)) for r in rows], dtype=torch.int32).reshape(len(rows), width)
        return table.to(device), torch.tensor([self._length[s] for s in seqs], dtype=torch.int32).to(device)
