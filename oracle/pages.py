"""Pages of the paged cache, step by step: rows that become other rows, pages for new tokens, kept tokens moved together.

TEST INFRASTRUCTURE ONLY (see the package docstring).  refs[p] is the number of table entries that are page p.

Pins: ``tests/test_drafts_oracle.py``.
"""
from __future__ import annotations

import numpy as np

from .cache import encode, scale_of
from .fp8 import decode_fp8


def counts(table, pages: int) -> np.ndarray:
    return np.bincount(table[table >= 0], minlength=pages)


def fork(table, lens, refs, source, size: int, window: int, sinks: int):
    """(table, lens, refs) after the rows have become their sources; source None: every row stays."""
    rows, width = table.shape
    new, new_lens = np.full_like(table, -1), np.zeros_like(lens)
    for s in range(rows):
        x = s if source is None else int(source[s])
        if not 0 <= x < rows:
            continue
        n = new_lens[s] = lens[x]
        for c in range(width):
            j = np.arange(c * size, (c + 1) * size)     # the places of this page; the next token is at position n
            if c * size < n and ((n - j < window) | (j < sinks)).any():
                new[s, c] = table[x, c]
    return new, new_lens, refs + counts(new, len(refs)) - counts(table, len(refs))


def reserve(table, lens, refs, cu, size: int):
    """(table, refs, pairs, missing): sequence by sequence, place by place."""
    table, refs = table.copy(), refs.copy()
    before = table.copy(), refs.copy()
    pairs = np.full((len(lens), 2), -1, dtype=np.int32)
    free = [int(p) for p in np.flatnonzero(refs == 0)]
    short = 0
    for s in range(len(lens)):
        count, n = int(cu[s + 1]) - int(cu[s]), int(lens[s])
        first = max(0, n - count)
        if count <= 0 or n <= 0:
            continue
        for c in range(first // size, (n - 1) // size + 1):
            if c >= table.shape[1]:
                break
            old = int(table[s, c])
            if old >= 0 and refs[old] == 1:
                continue
            if old >= 0:
                refs[old] -= 1
            if not free:
                short += 1
                continue
            new = free.pop(0)
            if old >= 0 and c * size < first:
                pairs[s] = old, new
            table[s, c], refs[new] = new, 1
    if short:
        return before[0], before[1], np.full_like(pairs, -1), short
    return table, refs, pairs, 0


def compact(codes, scales, table, target, keep, cu, first) -> None:
    """Codes [pages, H, size, d] and scales [pages, H] after the kept tokens have moved, in place."""
    size, pages = codes.shape[2], len(codes)

    def page_of(rows, s, place):
        c = place // size
        return int(rows[s, c]) if 0 <= place and c < rows.shape[1] and 0 <= rows[s, c] < pages else -1

    held, was = codes.copy(), scales.copy()
    where = {}
    for s in range(len(first)):
        for i in range(int(cu[s + 1]) - int(cu[s])):
            place = max(0, int(first[s])) + i
            to = page_of(target, s, place)
            if to >= 0:
                src = int(keep[int(cu[s]) + i])
                where.setdefault(to, []).append((place % size, page_of(table, s, src), src % size))
    for to, tokens in where.items():
        kept = min(slot for slot, _, _ in tokens)
        for h in range(codes.shape[1]):
            val = [decode_fp8(held[p, h, x]) * float(was[p, h]) if p >= 0 else np.zeros(codes.shape[3]) for _, p, x in tokens]
            fin = [np.abs(v[np.isfinite(v)]).max(initial=0.0) for v in val]
            new = scale_of(max(fin))
            if kept:
                old = float(was[to, h])
                if old > new:
                    new = old
                elif old < new:
                    codes[to, h, :kept] = encode(decode_fp8(held[to, h, :kept]) * (old / new))
            scales[to, h] = new
            for (slot, p, x), v in zip(tokens, val):
                same = p >= 0 and float(was[p, h]) == new
                codes[to, h, slot] = held[p, h, x] if same else encode(v / new)
