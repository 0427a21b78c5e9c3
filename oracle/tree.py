"""Trees of drafted tokens: masks and positions, and attention over the paged cache in fp64, from the definitions.

TEST INFRASTRUCTURE ONLY (see the package docstring).

* A drafted token's mask names itself and those that it follows, directly or not; its position is the number of tokens
  before it on its own path.
* A row at position p sees the tokens at places j before the drafted ones with p - j < window or j < sinks, and a drafted
  token at position y that its mask names with p - y < window or y < sinks; a row at a position below 0 sees nothing.  A
  window of 2^31 - 1 ends nothing.

Pins: ``tests/test_drafts_oracle.py``.
"""
from __future__ import annotations

import numpy as np

from .fp8 import decode_fp8
from .window import FP32, HALF_BF16


def masks(parents, cu, lens, words: int):
    """(named [total, 64 words] bool, positions [total])"""
    total = int(cu[-1])
    named, positions = np.zeros((total, 64 * words), dtype=bool), np.full(total, -1, dtype=np.int64)
    for s in range(len(lens)):
        t0, n = int(cu[s]), int(cu[s + 1]) - int(cu[s])
        for j in range(min(n, 64 * words)):
            path, at = [j], int(parents[t0 + j])
            while 0 <= at < path[-1]:
                path.append(at)
                at = int(parents[t0 + at])
            named[t0 + j, path] = True
            positions[t0 + j] = int(lens[s]) - n + len(path) - 1
    return named, positions


def words_of(named) -> np.ndarray:
    """named [total, 64 words] as int64 [total, words], bit j % 64 of word j / 64."""
    return np.packbits(named, axis=1, bitorder="little").view(np.int64)


def visible(n, count, named, positions, t0, t, window, sinks, capacity):
    """Places of a sequence of n tokens, `count` of them drafted (its first is row t0), that row t sees."""
    base, p = n - count, int(positions[t])
    if p < 0:
        return np.zeros(0, dtype=np.int64)
    j = np.arange(max(0, min(n, capacity)))
    x = j - base
    drafted = x >= 0
    ok = ~drafted
    inside = drafted & (x < named.shape[1])
    ok[inside] = named[t, x[inside]]
    place = np.where(drafted, positions[t0 + np.clip(x, 0, max(count - 1, 0))], j)
    return j[ok & ((p - place < window) | (place < sinks) | (window == 2 ** 31 - 1))]


def attention(q, codes_k, scale_k, codes_v, scale_v, table, lens, cu, named, positions, window: int, sinks: int, scale: float):
    """q [total, Hq, d] fp64 -> o, o_tol, lse, lse_tol (bounds as in oracle.cache)."""
    total, hq, d = q.shape
    size, hkv = codes_k.shape[2], codes_k.shape[1]
    o, o_tol = np.zeros(q.shape), np.zeros(q.shape)
    lse, lse_tol = np.full((hq, total), -np.inf), np.zeros((hq, total))
    for s in range(len(lens)):
        n, t0, count = max(0, int(lens[s])), int(cu[s]), int(cu[s + 1]) - int(cu[s])
        for t in range(t0, t0 + count):
            j = visible(n, count, named, positions, t0, t, window, sinks, table.shape[1] * size)
            page = table[s, j // size]
            ok = (page >= 0) & (page < len(codes_k))
            j, page = j[ok], page[ok]
            if not len(j):
                continue
            k = decode_fp8(codes_k[page, :, j % size]) * scale_k[page].astype(np.float64)[..., None]
            v = decode_fp8(codes_v[page, :, j % size]) * scale_v[page].astype(np.float64)[..., None]
            for h in range(hq):
                g = h // (hq // hkv)
                x = scale * (k[:, g] @ q[t, h])
                top = x.max()
                e = np.exp(x - top)
                prob = e / e.sum()
                o[t, h] = prob @ v[:, g]
                o_tol[t, h] = HALF_BF16 * np.abs(o[t, h]) + (HALF_BF16 + FP32) * (prob @ np.abs(v[:, g]))
                lse[h, t] = top + np.log(e.sum())
                lse_tol[h, t] = 2.0 ** -20 * (1 + abs(lse[h, t]) + d * scale * (np.abs(k[:, g]) @ np.abs(q[t, h])).max() / 16)
    return o, o_tol, lse, lse_tol
