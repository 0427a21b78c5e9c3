"""Index arithmetic of the window kernels (csrc/window.h, built for the host)."""
import numpy as np
import pytest

import oracle
import _window_host as H


@pytest.fixture(scope="module")
def host():
    return H.lib()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (5, 0), (7, 9), (20, 2), (31, 0), (31, 40), (100, 4)])
@pytest.mark.parametrize("first,rows", [(0, 90), (64, 64), (97, 33), (150, 70)])
def test_short_rows_read_what_some_query_sees(host, first, rows, window, sinks):
    # Rows `first` .. of a packed sequence in waves of 32; each forms delta of its short rows (fewer than 32 keys) from 64
    # positions around it and, where a document began further back, 32 of its first ones.
    lengths = [60, 1, 0, 30, 7, 2, 60, 1, 1, 58]
    cu = np.concatenate([[0], np.cumsum(lengths)])
    n = int(cu[-1])
    pos, keys = np.arange(first, first + rows), np.arange(n)
    ok = oracle.window_allowed(cu, pos, keys, window, sinks)
    seen = ok.any(0)
    start = cu[np.searchsorted(cu, pos, side="right") - 1]
    last = first + rows - 1
    read_elsewhere = 0
    for w in range(0, rows, 32):
        row = np.arange(w, min(w + 32, rows))
        short = row[ok[row].sum(1) < 32]
        if not len(short):
            continue
        g0, far = int(pos[w]), int(start[w])
        win = np.maximum(start, pos - (window - 1))
        held = np.minimum(sinks, win - start)
        lo = int(win[short[0]])
        of_far = short[start[short] == far]
        far_end = far + int(held[of_far[-1]]) if len(of_far) else far
        got = set()
        for j0 in (g0 - 32, g0, far):
            for x in range(j0, j0 + 32):
                key = host.short_row(x, g0, lo, far, far_end, last)
                assert 0 <= key < n and seen[key], (w, x, key)      # rows that no query sees are not read
                read_elsewhere += key != x
                if key == x:
                    got.add(x)
        for i in short:                                             # and every key of a short row is
            assert set(keys[ok[i]]) <= got, (w, i)
    assert read_elsewhere
