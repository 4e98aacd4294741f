"""The paged cache of ciphertext rows, one row at a time (CPU oracle; test
infrastructure only).

Sequences of rows live in pages that several sequences may hold (the encrypted
K/V cache of section 4.1's KV backends).  Every call is written as the plain loop
over its requests; which requests are bad is decided from the call's lists
before anything changes, as the interface states it.

Parity: pinned (tests/test_oracle_cache.py) against plain Python lists of rows, one
list a sequence, through random runs of all calls.
"""
from __future__ import annotations

import numpy as np

OK, BAD_REQUEST, TABLE_FULL, NO_PAGES = range(4)


class Cache:
    def __init__(self, pages: int, page_rows: int, row_shape: tuple, seqs: int, max_pages: int):
        self.pool = np.zeros((pages, page_rows) + tuple(row_shape), dtype=np.uint32)
        self.refs = np.zeros(pages, dtype=np.int32)
        self.table = np.full((seqs, max_pages), -1, dtype=np.int32)
        self.lens = np.zeros(seqs, dtype=np.int32)

    @property
    def page_rows(self) -> int:
        return self.pool.shape[1]

    def _known(self, s) -> bool:
        return 0 <= s < len(self.lens)

    def _pages(self, rows: int) -> int:
        return -(-int(rows) // self.page_rows)

    def _shorten(self, s: int, keep: int) -> None:
        for at in range(self._pages(keep), self._pages(self.lens[s])):
            self.refs[self.table[s, at]] -= 1
            self.table[s, at] = -1
        self.lens[s] = min(keep, self.lens[s])

    def free(self, seq, keep=None) -> list:
        seq = [int(s) for s in seq]
        status = [OK if self._known(s) and seq.count(s) == 1 else BAD_REQUEST for s in seq]
        for i, s in enumerate(seq):
            if status[i] == OK:
                self._shorten(s, 0 if keep is None else max(0, int(keep[i])))
        return status

    def fork(self, src, dst) -> list:
        src, dst = [int(s) for s in src], [int(d) for d in dst]
        status = []
        for i, (s, d) in enumerate(zip(src, dst)):
            fine = self._known(s) and self._known(d) and dst.count(d) == 1 and d not in src and s not in dst
            status.append(OK if fine else BAD_REQUEST)
        for i, (s, d) in enumerate(zip(src, dst)):
            if status[i] == OK:
                self._shorten(d, 0)
                self.table[d], self.lens[d] = self.table[s], self.lens[s]
                for page in self.table[d, : self._pages(self.lens[d])]:
                    self.refs[page] += 1
        return status

    def append(self, seq, rows, row0=None) -> list:
        seq = [int(s) for s in seq]
        count, n = len(seq), len(rows)
        if row0 is None:
            spans = [(i, i + 1) if i < n else None for i in range(count)]
            astray = False
        else:
            spans = [(int(row0[i]), int(row0[i + 1])) for i in range(count)]
            astray = any(a < 0 or b < a or b > n for a, b in spans)
        status = []
        for s, span in zip(seq, spans):
            if astray or span is None or not self._known(s) or seq.count(s) != 1:
                status.append(BAD_REQUEST)
            elif self.lens[s] + span[1] - span[0] > self.table.shape[1] * self.page_rows:
                status.append(TABLE_FULL)
            else:
                status.append(OK)
        before = [a.copy() for a in (self.pool, self.refs, self.table, self.lens)]
        keepers = self._keepers(seq, [range(*span) if st == OK else () for span, st in zip(spans, status)])
        try:
            for i, (s, span, st) in enumerate(zip(seq, spans, status)):
                if st == OK:
                    for r in range(*span):
                        self._append_row(s, rows[r], i in keepers)
        except IndexError:  # no free page left: the call leaves the cache as it was
            self.pool, self.refs, self.table, self.lens = before
            status = [NO_PAGES if st == OK else st for st in status]
        return status

    def _keepers(self, seq, new_rows) -> set:
        """Requests that write their last page in place though others hold it: where all of its holders
        append, the one with the most rows on it, of those the last."""
        writers = {}
        for i, (s, r) in enumerate(zip(seq, new_rows)):
            if len(r) and self.lens[s] % self.page_rows:
                page = int(self.table[s, self.lens[s] // self.page_rows])
                writers.setdefault(page, []).append((int(self.lens[s] % self.page_rows), i))
        return {max(w)[1] for page, w in writers.items() if len(w) == self.refs[page]}

    def _append_row(self, s: int, row, keeps: bool) -> None:
        at, slot = divmod(int(self.lens[s]), self.page_rows)
        page = self.table[s, at] if slot else -1
        if page < 0 or (self.refs[page] > 1 and not keeps):
            fresh = np.flatnonzero(self.refs == 0)[0]
            if page >= 0:
                self.pool[fresh, :slot] = self.pool[page, :slot]
                self.refs[page] -= 1
            self.refs[fresh] = 1
            self.table[s, at] = page = fresh
        self.pool[page, slot] = row
        self.lens[s] += 1

    def compact(self) -> int:
        live = int(np.sum(self.refs > 0))
        for page in range(live, len(self.refs)):
            if self.refs[page] > 0:
                hole = np.flatnonzero(self.refs == 0)[0]
                self.pool[hole] = self.pool[page]
                self.refs[hole], self.refs[page] = self.refs[page], 0
                self.table[self.table == page] = hole
        return live

    def gather(self, seq, pos) -> np.ndarray:
        out = np.zeros((len(seq),) + self.pool.shape[2:], dtype=np.uint32)
        for r, (s, p) in enumerate(zip(seq, pos)):
            if self._known(s) and 0 <= p < self.lens[s]:
                out[r] = self.pool[self.table[s, p // self.page_rows], p % self.page_rows]
        return out
