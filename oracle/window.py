"""Window attention with sinks on packed documents, in fp64, from its definition, with how far a result in limited
precision may be off.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Query at position i of a document that starts at s sees key j iff s <= j <= i and (i - j < window or j - s < sinks).

The error bounds are per element and count roundings.  A bf16 value is off by at most half a step, 2^-8 of itself;
P and dS are rounded to bf16 before their products, outputs when stored.  fp32 work (sums of a few thousand terms,
exponentials, the recomputed P from a stored LSE) is covered by 2^-12 of the sum of absolute terms: a score of
size s rounds by d s 2^-24 and its exponential by about 2^-21 |s|, below 2^-12 for the |s| < 100 of these tests.

Pins (``tests/test_window_oracle.py``): brute force over pairs, the packed causal oracle for a window that ends
nothing, finite differences.
"""
from __future__ import annotations

from typing import Dict

import numpy as np

HALF_BF16 = 2.0 ** -8
FP32 = 2.0 ** -12


def window_allowed(cu_seqlens, positions, keys, window: int, sinks: int) -> np.ndarray:
    """Boolean [queries, keys]."""
    cu = np.asarray(cu_seqlens, dtype=np.int64)
    i, j = np.asarray(positions)[:, None], np.asarray(keys)[None]
    start = cu[np.searchsorted(cu, np.asarray(positions), side="right") - 1][:, None]
    return (j >= start) & (j <= i) & ((i - j < window) | (j - start < sinks)) & (i < cu[-1])


def window_attention(q, k, v, cu_seqlens, positions, window: int, sinks: int, scale: float, d_o=None) -> Dict:
    """q [n, Hq, d] at global `positions`; k, v [N, Hkv, d] in global order.  Returns o, lse and, with d_o, dq, dk, dv
    (this call's queries' share of every key), each with a bound `<name>_tol` on the error of a bf16 result (lse:
    fp32).  Rows of queries behind the last document are 0 (lse: -inf)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n, hq, d = q.shape
    hkv = k.shape[1]
    ok = window_allowed(cu_seqlens, positions, np.arange(k.shape[0]), window, sinks)
    out = {name: np.zeros(q.shape) for name in ("o", "o_tol")}
    out["lse"], out["lse_tol"] = np.full((hq, n), -np.inf), np.zeros((hq, n))
    if d_o is not None:
        d_o = np.asarray(d_o, dtype=np.float64)
        for name in ("dq", "dq_tol"):
            out[name] = np.zeros(q.shape)
        for name in ("dk", "dv", "dk_tol", "dv_tol"):
            out[name] = np.zeros(k.shape)
    live = ok.any(1)
    for h in range(hq):
        g = h // (hq // hkv)
        s = np.where(ok, scale * (q[:, h] @ k[:, g].T), -np.inf)[live]
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        den = p.sum(1, keepdims=True)
        p /= den
        lse = (top + np.log(den))[:, 0]
        o = p @ v[:, g]
        mass = p @ np.abs(v[:, g])
        o_tol = HALF_BF16 * np.abs(o) + (HALF_BF16 + FP32) * mass
        out["o"][live, h], out["o_tol"][live, h] = o, o_tol
        size = scale * (np.abs(q[live, h]) @ np.abs(k[:, g]).T).max(1)
        out["lse"][h, live], out["lse_tol"][h, live] = lse, 2.0 ** -20 * (1 + np.abs(lse) + d * size / 16)
        if d_o is None:
            continue
        do = d_o[live, h]
        dp = do @ v[:, g].T
        delta = (do * o).sum(1, keepdims=True)
        ds = p * (dp - delta)
        # dS: its own rounding, delta taken from the rounded O, fp32 work
        ds_tol = HALF_BF16 * np.abs(ds) + p * ((np.abs(do) * o_tol).sum(1, keepdims=True)
                                               + FP32 * (np.abs(do) @ np.abs(v[:, g]).T + (np.abs(do) * mass).sum(1, keepdims=True)))
        dq, dk, dv = scale * ds @ k[:, g], scale * ds.T @ q[live, h], p.T @ do
        out["dq"][live, h] = dq
        out["dq_tol"][live, h] = HALF_BF16 * np.abs(dq) + scale * ((ds_tol + FP32 * np.abs(ds)) @ np.abs(k[:, g]))
        out["dk"][:, g] += dk
        out["dv"][:, g] += dv
        out["dk_tol"][:, g] += scale * ((ds_tol + FP32 * np.abs(ds)).T @ np.abs(q[live, h]))
        out["dv_tol"][:, g] += (HALF_BF16 + FP32) * (p.T @ np.abs(do))
    if d_o is not None:
        out["dk_tol"] += HALF_BF16 * np.abs(out["dk"])
        out["dv_tol"] += HALF_BF16 * np.abs(out["dv"])
    return out
