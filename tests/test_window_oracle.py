"""Pins of the fp64 oracle of window attention with sinks: brute force over pairs, the packed causal oracle for a window
that ends nothing, finite differences for the gradients."""
import math

import numpy as np
import pytest

import oracle


def _inputs(n, hq, hkv, d, seed=0):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((n, hq, d)), rng.standard_normal((n, hkv, d)), rng.standard_normal((n, hkv, d)), \
        rng.standard_normal((n, hq, d))


@pytest.mark.parametrize("cu,window,sinks", [([0, 9], 3, 0), ([0, 4, 4, 9], 2, 1), ([0, 1, 8], 1, 3), ([0, 5, 7], 4, 9)])
def test_allowed_pairs_by_brute_force(cu, window, sinks):
    n = 9
    got = oracle.window_allowed(cu, np.arange(n), np.arange(n), window, sinks)
    for i in range(n):
        doc = [(a, b) for a, b in zip(cu, cu[1:]) if a <= i < b]
        for j in range(n):
            want = False
            if doc:
                a, b = doc[0]
                want = a <= j <= i and (j > i - window or j < a + sinks)
            assert got[i, j] == want, (i, j)


def test_wide_window_is_the_packed_causal_attention():
    cu = [0, 7, 7, 20, 33]
    q, k, v, do = _inputs(33, 4, 2, 16)
    got = oracle.window_attention(q, k, v, cu, np.arange(33), 33, 0, 1 / math.sqrt(16), do)
    want = oracle.shard_forward(q, k, v, cu, 33, 1, "contiguous", 0)
    assert np.allclose(got["o"], want["o"], atol=1e-12) and np.allclose(got["lse"], want["lse"], atol=1e-12)


@pytest.mark.parametrize("window,sinks", [(3, 0), (2, 2), (1, 1), (50, 4)])
def test_gradients_by_differences(window, sinks):
    cu, scale = [0, 6, 17], 0.3
    q, k, v, do = _inputs(17, 2, 1, 5, seed=3)
    pos = np.arange(17)
    ref = oracle.window_attention(q, k, v, cu, pos, window, sinks, scale, do)

    def loss():
        return (oracle.window_attention(q, k, v, cu, pos, window, sinks, scale)["o"] * do).sum()

    rng = np.random.default_rng(5)
    for x, name in ((q, "dq"), (k, "dk"), (v, "dv")):
        for _ in range(12):
            at = tuple(rng.integers(0, m) for m in x.shape)
            old, eps = x[at], 1e-5
            x[at] = old + eps
            up = loss()
            x[at] = old - eps
            down = loss()
            x[at] = old
            assert abs((up - down) / (2 * eps) - ref[name][at]) < 1e-8, (name, at)
