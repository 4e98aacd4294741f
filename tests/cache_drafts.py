"""Calls on a cache as speculative decoding makes them: prompts forked into
branches, branches cut back to lengths of their own, and then branches and prompt
appended to together, so that one page has holders of unlike lengths."""
from __future__ import annotations

import numpy as np

SEQS = 9


def calls(rng, rounds: int, page_rows: int):
    """(name, arguments) of one call at a time: ("append", seq, counts), ("fork", src, dst), ("free", seq, keep),
    ("compact",)."""
    for _ in range(rounds):
        holders = rng.permutation(SEQS)[: rng.integers(2, 6)].tolist()
        yield "free", list(range(SEQS)), None
        other = next(s for s in range(SEQS) if s not in holders)
        length = int(rng.integers(1, 3 * page_rows + 1))
        yield "append", [other, holders[0]], [int(rng.integers(0, 2 * page_rows)), length]
        yield "fork", [holders[0]] * (len(holders) - 1), holders[1:]
        page0 = (length - 1) // page_rows * page_rows
        cut = [s for s in holders if rng.integers(2)]
        yield "free", cut, [int(rng.integers(page0 + 1, length + 1)) for _ in cut]
        if rng.integers(3) == 0:
            yield "free", [other], None
            yield ("compact",)
        who = rng.permutation(holders).tolist()
        if rng.integers(4) == 0:
            who.pop()                                  # one holder does not append, so all copy
        counts = rng.integers(1, page_rows + 2, len(who))
        if rng.integers(5) == 0:
            counts[rng.integers(len(who))] = 0
        yield "append", who + [other], counts.tolist() + [int(rng.integers(0, 3))]


def shared_last_pages(lens, table, refs, page_rows, seq, counts):
    """Of an append's served requests: (pages whose holders all append, those of them with holders of unlike lengths)."""
    parts = {}
    for s, n in zip(seq, counts):
        at, part = divmod(int(lens[s]), page_rows)
        if n and part and refs[table[s, at]] > 1:
            parts.setdefault(int(table[s, at]), []).append(part)
    kept = [v for page, v in parts.items() if len(v) == refs[page]]
    return len(kept), sum(len(set(v)) > 1 for v in kept)


def clashes(lens, table, now, page_rows, seq, counts):
    """Slots (page, row) that an append both copies for one request and writes for another, from the tables
    before it and after: its moves run in no order, so there may be none."""
    copied, written = set(), set()
    for s, n in zip(seq, counts):
        at, part = divmod(int(lens[s]), page_rows)
        if n and part:
            page = int(table[s, at])
            if now[s, at] == page:
                written |= {(page, k) for k in range(part, min(page_rows, part + n))}
            else:
                copied |= {(page, k) for k in range(part)}
    return copied & written
