"""The paged 8-bit K/V cache: what an append leaves in it, and attention over it in fp64, from the definitions.

TEST INFRASTRUCTURE ONLY (see the package docstring).

* Rotation of a pair (a, b) by (cos, sin) of its position: (a cos - b sin, b cos + a sin), pairs (i, i + rot / 2) or
  (2 i, 2 i + 1).
* The scale of a page and head is 2^e, e the smallest exponent in -100..120 with 448 * 2^e >= every finite value; code =
  e4m3(value / scale), nearest even, saturating.  A page that held tokens before keeps at least its scale; if it
  grows, the older codes become e4m3(code * old / new).
* A query at position p sees the tokens j <= p with p - j < window or j < sinks.

Pins: ``tests/test_cache_oracle.py``.
"""
from __future__ import annotations

import numpy as np
import torch

from .fp8 import decode_fp8
from .window import FP32, HALF_BF16


def rotate(x, rows, interleaved: bool, dtype=np.float64) -> np.ndarray:
    """x [..., d] by rows [..., rot] (cos | sin), broadcast over the heads; `dtype` float32 rounds every operation."""
    x, rows = np.asarray(x).astype(dtype), np.asarray(rows).astype(dtype)
    rot = rows.shape[-1]
    out = x.copy()
    if rot == 0:
        return out
    cos, sin = rows[..., :rot // 2], rows[..., rot // 2:]
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    out[..., a] = x[..., a] * cos - x[..., b] * sin
    out[..., b] = x[..., b] * cos + x[..., a] * sin
    return out


def scale_of(amax) -> float:
    e = -100
    while e < 120 and 448.0 * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


def encode(x) -> np.ndarray:
    y = np.clip(np.asarray(x, dtype=np.float32), -448, 448)
    return torch.from_numpy(np.ascontiguousarray(y)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def append(codes, scales, table, positions, values) -> None:
    """values fp32 [tokens, H, d] at the given (sequence, position) pairs into codes [pages, H, size, d] and scales
    [pages, H], in place; tokens of one call, each sequence's in order."""
    size = codes.shape[2]
    where = {}
    for t, (s, p) in enumerate(positions):
        if 0 <= p < table.shape[1] * size and 0 <= table[s, p // size] < len(codes):
            where.setdefault(int(table[s, p // size]), []).append((p % size, t))
    for page, tokens in where.items():
        held = min(slot for slot, _ in tokens)
        for h in range(codes.shape[1]):
            val = np.stack([values[t, h] for _, t in tokens])
            fin = np.abs(val[np.isfinite(val)])
            new = scale_of(fin.max(initial=0.0))
            if held:
                old = float(scales[page, h])
                if old > new:
                    new = old
                elif old < new:
                    again = decode_fp8(codes[page, h, :held]) * (old / new)
                    codes[page, h, :held] = encode(again)
            scales[page, h] = new
            for (slot, _), x in zip(tokens, val):
                codes[page, h, slot] = encode(x / np.float32(new))


def attention(q, codes_k, scale_k, codes_v, scale_v, table, lens, cu, window: int, sinks: int, scale: float):
    """q [total, Hq, d] fp64 -> o, o_tol, lse, lse_tol (bounds as in oracle.window)."""
    total, hq, d = q.shape
    size, hkv = codes_k.shape[2], codes_k.shape[1]
    o, o_tol = np.zeros(q.shape), np.zeros(q.shape)
    lse, lse_tol = np.full((hq, total), -np.inf), np.zeros((hq, total))
    for s in range(len(lens)):
        n = int(lens[s])
        for t in range(int(cu[s]), int(cu[s + 1])):
            p = n - int(cu[s + 1]) + t
            j = np.arange(max(0, min(p + 1, table.shape[1] * size)))
            j = j[(p - j < window) | (j < sinks)]
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
