"""Which pages of a paged cache belong to which sequences, kept on the host: sequences are added, extended, forked and freed, and pages
shared by forks are copied when one of them goes on writing. No tensors here; PagedCache runs the copies."""
from __future__ import annotations

import math

import numpy as np


class PageTable:
    """Sequences are numbered 0 .. sequences - 1 (rows of ``table``); ``lengths`` holds their tokens. A page may belong to several
    sequences (``refs`` counts them); tokens are only ever written to pages of one."""

    def __init__(self, pages: int, page_size: int, sequences: int, width: int):
        if pages < 0 or sequences < 1 or width < 1:
            raise ValueError("a cache needs pages >= 0, and at least one sequence and one page a sequence")
        if page_size < 16 or page_size > 65536 or page_size & (page_size - 1):
            raise ValueError(f"page_size must be a power of two from 16 to 65536, got {page_size}")
        self.page_size = page_size
        self.table = np.full((sequences, width), -1, dtype=np.int32)
        self.lengths = np.zeros(sequences, dtype=np.int32)
        self.counts = np.zeros(sequences, dtype=np.int32)  # pages of each sequence: those of its tokens, and reserved ones
        self.room = np.zeros(sequences, dtype=np.int64)  # tokens that may follow each sequence's: reserved, and in pages of its own
        self.active = np.zeros(sequences, dtype=bool)
        self.refs = np.zeros(pages, dtype=np.int32)
        self._free = list(range(pages - 1, -1, -1))

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def add(self) -> int:
        """A new, empty sequence's number."""
        idle = np.flatnonzero(~self.active)
        if idle.size == 0:
            raise RuntimeError(f"all {self.active.size} sequences are in use")
        s = int(idle[0])
        self.active[s] = True
        return s

    def _rows(self, sequences, tokens):
        rows, more = np.atleast_1d(np.asarray(sequences)), np.asarray(tokens)
        for x in (rows, more):
            if x.size and (x.dtype.kind not in "iu" or x.max() >= 2 ** 31):
                raise ValueError("sequences and tokens must be whole numbers below 2^31")
        rows, more = rows.astype(np.int64), more.astype(np.int64)
        more = np.broadcast_to(more, rows.shape)
        if rows.ndim != 1 or np.unique(rows).size != rows.size:
            raise ValueError("sequences must be a list of different numbers")
        if rows.size and (rows.min() < 0 or rows.max() >= self.active.size or not self.active[rows].all()):
            raise ValueError("a sequence is not in use")
        if (more < 0).any():
            raise ValueError("tokens must be >= 0")
        return rows, more

    def reserve(self, sequences, tokens):
        """Makes room for so many more tokens in each sequence without adding them; returns the pages to copy first (src, dst): those
        that the next tokens go to and that others share. The room lasts until the sequence is forked or truncated: its next tokens may go
        to a page that others share then. Raises without a change if pages or the table do not suffice."""
        rows, more = self._rows(sequences, tokens)
        new = self.lengths[rows].astype(np.int64) + more
        want = -(-new // self.page_size)
        if (want > self.table.shape[1]).any():
            raise RuntimeError(f"a sequence of {int(new.max())} tokens passes its {self.table.shape[1]} pages of {self.page_size}")
        fresh = np.maximum(want - self.counts[rows], 0)
        # The begun page that the next token goes to, where others share it. (Full pages are not written again, and reserved ones are not
        # shared.) Of several that share it here, the last to be seen keeps it if none outside does.
        split, left = [], {}
        for s, n in zip(rows.tolist(), more.tolist()):
            j, begun = divmod(int(self.lengths[s]), self.page_size)
            if n == 0 or begun == 0:
                continue
            page = int(self.table[s, j])
            refs = left.get(page, int(self.refs[page]))
            if refs > 1:
                split.append((s, j, page))
                left[page] = refs - 1
        need = int(fresh.sum()) + len(split)
        if need > len(self._free):
            raise RuntimeError(f"{need} pages are needed, {len(self._free)} are free")
        src, dst = [], []
        for s, j, page in split:
            to = self._take()
            src.append(page)
            dst.append(to)
            self.refs[page] -= 1
            self.table[s, j] = to
        for s, n in zip(rows.tolist(), fresh.tolist()):
            for _ in range(n):
                self.table[s, self.counts[s]] = self._take()
                self.counts[s] += 1
        self.room[rows] = np.maximum(self.room[rows], more)
        return np.array(src, dtype=np.int32), np.array(dst, dtype=np.int32)

    def _take(self) -> int:
        page = self._free.pop()
        self.refs[page] = 1
        return page

    def extend(self, sequences, tokens):
        """reserve(), with the tokens added to the lengths."""
        pairs = self.reserve(sequences, tokens)
        self.grown(sequences, tokens)
        return pairs

    def grown(self, sequences, tokens) -> None:
        """Tokens that were added in room reserved before."""
        rows, more = self._rows(sequences, tokens)
        if (more > self.room[rows]).any():
            raise ValueError("more tokens than were reserved (a fork or truncation ends the room)")
        self.room[rows] -= more
        self.lengths[rows] += more.astype(np.int32)

    def offsets(self, tokens):
        """int32 offsets of a call in which sequence s has tokens[s] new tokens (a dict, or one count for each sequence)."""
        counts = np.zeros(self.active.size, dtype=np.int64)
        size = counts.size
        for s, n in tokens.items() if isinstance(tokens, dict) else enumerate(tokens):
            if not 0 <= s < size or not 0 <= n < 2 ** 31 or s % 1:
                raise ValueError(f"{n} tokens of sequence {s}, of {size}")
            counts[s] = n
        cu = np.concatenate([[0], np.cumsum(counts)])
        if math.fsum(tokens.values() if isinstance(tokens, dict) else tokens) != cu[-1]:  # what is stored of a fraction is less
            raise ValueError(f"numbers of tokens must be whole, got {tokens}")
        if cu[-1] >= 2 ** 31:
            raise ValueError(f"{cu[-1]} tokens are too many for one call")
        return cu.astype(np.int32)

    def fork(self, sequence: int) -> int:
        """A new sequence with the same tokens, whose pages both share."""
        (s,), _ = self._rows([sequence], 0)
        t = self.add()
        n = -(-int(self.lengths[s]) // self.page_size)  # not the reserved ones
        self.table[t, :n] = self.table[s, :n]
        self.refs[self.table[s, :n]] += 1
        self.counts[t], self.lengths[t] = n, self.lengths[s]
        self.room[s] = 0
        return t

    def free(self, sequence: int) -> None:
        """Ends a sequence; pages that no other one has are free again."""
        (s,), _ = self._rows([sequence], 0)
        self._drop(s, 0)
        self.active[s] = False
        self.lengths[s] = 0

    def truncate(self, sequence: int, tokens: int) -> None:
        """Takes a sequence back to its first tokens (as when proposed ones are rejected)."""
        (s,), _ = self._rows([sequence], 0)
        if not 0 <= tokens <= self.lengths[s]:
            raise ValueError(f"sequence {sequence} has {self.lengths[s]} tokens")
        self._drop(s, -(-tokens // self.page_size))
        self.lengths[s] = tokens

    def _drop(self, s, keep) -> None:
        pages = self.table[s, keep:self.counts[s]]
        self.refs[pages] -= 1
        self._free.extend(int(p) for p in pages[::-1] if self.refs[p] == 0)
        self.table[s, keep:self.counts[s]] = -1
        self.counts[s] = keep
        self.room[s] = 0

    def compact(self):
        """Moves pages so that those in use are the first ones; returns the copies (src, dst) that carry them out."""
        used = np.flatnonzero(self.refs > 0)
        n = used.size
        src = used[used >= n].astype(np.int32)
        dst = np.flatnonzero(self.refs[:n] == 0).astype(np.int32)
        to = np.arange(self.refs.size, dtype=np.int32)
        to[src] = dst
        held = self.table >= 0
        self.table[held] = to[self.table[held]]
        self.refs[dst] = self.refs[src]
        self.refs[src] = 0
        self._free = list(range(self.refs.size - 1, n - 1, -1))
        return src, dst
