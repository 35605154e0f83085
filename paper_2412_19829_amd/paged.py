"""A paged key-value cache: which sequence holds which pages (host), and the tensors that the library's
entry points take (device).

A sequence's row of `table` lists its pages, `lens` its tokens.  Pages are counted by the sequences that hold them: a
fork shares the full ones, which nobody writes again, and takes a copy of the last one if that is partly filled.
Every change of the bookkeeping is checked before it is made, so a refused call leaves the cache as it was.
The copies run on torch's current stream, in order with what changes of `table` and `lens`, and no call waits for it: a program that
uses the cache on another stream has that one wait.  The books do not change while a graph is captured.
reserve() and advance() for one token of every sequence take the host, us, without a new page / with one for each: 32 sequences 32 / 100, 256 152 / 240,
however many pages a row has (with the whole table sent each time, 256 rows of 2048 took 12500 / 25000).
"""
from __future__ import annotations

import torch

from . import binding as gb


class PagedCache:
    """Room for `n_pages` pages of `page_size` tokens, for up to `max_seqs` sequences of up to `max_pages` pages, `n_heads` key
    heads of size `d` in each of `layers` layers."""

    def __init__(self, n_pages: int, page_size: int, n_heads: int, d: int, max_seqs: int, max_pages: int, *, layers: int = 1,
                 dtype=torch.bfloat16, device="cuda"):
        if min(n_pages, page_size, n_heads, d, max_seqs, max_pages, layers) < 1:
            raise ValueError("sizes must be positive")
        if d not in (64, 128) or dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("d is 64 or 128, dtype bfloat16 or float32")
        if not 8 <= page_size <= 65536 or page_size & (page_size - 1) or max_pages * page_size > 1 << 30:
            raise ValueError("page_size is a power of two from 8 to 65536, a sequence has at most 2^30 tokens")
        self.page_size, self.n_heads, self.max_pages = page_size, n_heads, max_pages
        self.kpages = torch.zeros(n_pages, layers * n_heads, page_size, d, dtype=dtype, device=device)
        self.vpages = torch.zeros_like(self.kpages)
        self.table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device)
        self.lens = torch.full((max_seqs,), -1, dtype=torch.int32, device=device)   # -1: an idle row
        self._held = [0] * n_pages                         # sequences that hold the page
        self._free = list(range(n_pages - 1, -1, -1))      # the lowest last: taken first
        self._pages = [None] * max_seqs                    # per sequence; None: no such sequence
        self._len = [-1] * max_seqs

    def layer(self, i: int):
        """(kpages, vpages) of one layer, as views."""
        heads = slice(i * self.n_heads, (i + 1) * self.n_heads)
        return self.kpages[:, heads], self.vpages[:, heads]

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, seq: int) -> int:
        self._check(seq)
        return self._len[seq]

    def pages(self, seq: int) -> list:
        self._check(seq)
        return list(self._pages[seq])

    def _check(self, seq):
        if not 0 <= seq < len(self._pages) or self._pages[seq] is None:
            raise ValueError(f"no sequence {seq}")

    def _slot(self):
        for s, p in enumerate(self._pages):
            if p is None:
                return s
        raise RuntimeError("the cache holds as many sequences as it can")

    def _next(self, n):
        """The pages that _take() would take."""
        if n > len(self._free):
            raise RuntimeError(f"the cache is full: {n} pages wanted, {len(self._free)} free")
        return self._free[len(self._free) - n:][::-1]

    def _take(self, n):
        taken = self._next(n)
        del self._free[len(self._free) - n:]
        for p in taken:
            self._held[p] = 1
        return taken

    def _host(self, numbers, dtype):
        """Memory of their own for numbers on their way to the device, which a copy keeps until it has run (but not until it runs again)."""
        if self.table.is_cuda and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the books cannot change while a graph is captured: its replays would not change them")
        return torch.tensor(numbers, dtype=dtype, pin_memory=self.table.is_cuda)

    def _send(self, numbers, dtype):
        return self._host(numbers, dtype).to(self.table.device, non_blocking=True)

    def _update(self, lens, pages=()):
        """`lens` {sequence: tokens} and `pages` [(sequence, place in its row, page)], on the device and then in the books of lengths:
        where there is no memory for it, nothing has changed."""
        new = list(self._len)
        for s, n in lens.items():
            new[s] = n
        if pages:
            at = self._send([s * self.max_pages + i for s, i, _ in pages], torch.int64)
            values = self._send([p for _, _, p in pages], torch.int32)
        if lens:
            self.lens.copy_(self._host(new, torch.int32), non_blocking=True)
        if pages:
            self.table.view(-1).scatter_(0, at, values)
        self._len = new

    def _copy(self, pairs):
        if pairs:
            src, dst = self._send(list(zip(*pairs)), torch.int32)
            gb.gformer_pages_copy(self.kpages, self.vpages, src, dst)

    def open(self, tokens: int = 0) -> int:
        """A new sequence of `tokens` tokens, whose keys and values the caller writes (gformer_paged_fill)."""
        n = -(-tokens // self.page_size)
        if tokens < 0 or n > self.max_pages:
            raise ValueError(f"a sequence has 0 to {self.max_pages * self.page_size} tokens")
        seq = self._slot()
        self._update({seq: tokens}, [(seq, i, p) for i, p in enumerate(self._next(n))])
        self._pages[seq] = self._take(n)
        return seq

    def fork(self, seq: int) -> int:
        """A sequence that goes on from the same tokens."""
        self._check(seq)
        new, mine = self._slot(), self._pages[seq]
        partly = self._len[seq] % self.page_size != 0
        full = len(mine)
        if partly or full * self.page_size > self._len[seq]:
            full = self._len[seq] // self.page_size
        own = self._next(1 if partly else 0)
        if partly:
            self._copy([(mine[full], own[0])])
        pages = mine[:full] + own
        self._update({new: self._len[seq]}, [(new, i, p) for i, p in enumerate(pages)])
        self._take(len(own))
        for p in mine[:full]:
            self._held[p] += 1
        self._pages[new] = pages
        return new

    def free(self, seq: int) -> None:
        """Gives a sequence's pages back, as far as no other holds them."""
        self._check(seq)
        self._update({seq: -1}, [(seq, i, -1) for i in range(len(self._pages[seq]))])
        for p in self._pages[seq]:
            self._held[p] -= 1
            if self._held[p] == 0:
                self._free.append(p)
        self._free.sort(reverse=True)
        self._pages[seq] = None

    def reserve(self, seqs) -> None:
        """A slot for the next token of each of `seqs`: what a step needs before it writes."""
        seqs = list(dict.fromkeys(seqs))
        for s in seqs:
            self._check(s)
            if self._len[s] >= self.max_pages * self.page_size:
                raise ValueError(f"sequence {s} is as long as it can be")
        short = [s for s in seqs if len(self._pages[s]) * self.page_size == self._len[s]]
        if short:
            new = list(zip(short, self._next(len(short))))
            self._update({}, [(s, len(self._pages[s]), p) for s, p in new])
            self._take(len(short))
            for s, p in new:
                self._pages[s].append(p)

    def advance(self, seqs) -> None:
        """After a step that wrote one token of each of `seqs` in every layer."""
        seqs = list(dict.fromkeys(seqs))
        for s in seqs:
            self._check(s)
            if len(self._pages[s]) * self.page_size <= self._len[s]:
                raise ValueError(f"sequence {s} has no slot for the token: reserve() comes first")
        self._update({s: self._len[s] + 1 for s in seqs})

    def compact(self) -> int:
        """Moves the pages in use to the cache's front; returns how many were moved."""
        used = sorted(p for p, n in enumerate(self._held) if n)
        holes = [p for p in range(len(used)) if not self._held[p]]
        moved = dict(zip(used[len(used) - len(holes):], holes))
        self._copy(list(moved.items()))
        self._update({}, [(s, i, moved[p]) for s, pages in enumerate(self._pages) for i, p in enumerate(pages or ()) if p in moved])
        for old, new in moved.items():
            self._held[new], self._held[old] = self._held[old], 0
        for pages in self._pages:
            if pages:
                pages[:] = [moved.get(p, p) for p in pages]
        self._free = [p for p in range(len(self._held) - 1, -1, -1) if not self._held[p]]
        return len(moved)
