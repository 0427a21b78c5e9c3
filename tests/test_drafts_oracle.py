"""Pins of oracle.tree and oracle.pages: worked examples, and the oracles of what they must agree with."""
import numpy as np
import pytest

from oracle import cache as C
from oracle import pages as P
from oracle import tree as T
from oracle.fp8 import decode_fp8


def test_masks_of_a_worked_tree():
    # 0 - 1 - 3, 0 - 2, 4 (no parent), 5 follows 4; a second sequence with a parent that is none (its own number)
    named, positions = T.masks([-1, 0, 0, 1, -1, 4, -7, 1], [0, 6, 8], [106, 2], 1)
    want = [{0}, {0, 1}, {0, 2}, {0, 1, 3}, {4}, {4, 5}, {0}, {1}]
    assert [set(np.flatnonzero(r)) for r in named] == want
    assert positions.tolist() == [100, 101, 101, 102, 100, 101, 0, 0]
    assert T.words_of(named)[:, 0].tolist() == [1, 3, 5, 11, 16, 48, 1, 2]


def test_tokens_behind_the_mask():
    named, positions = T.masks(list(range(-1, 69)), [0, 70], [70], 1)
    assert named[63].all() and not named[64:].any() and positions[63] == 63 and (positions[64:] == -1).all()
    assert T.words_of(named)[63, 0] == -1


def _cache(lens, size, hkv, d, seed):
    rng = np.random.default_rng(seed)
    per = [-(-n // size) for n in lens]
    order = rng.permutation(sum(per) + 2)
    table = np.full((len(lens), max(per)), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(per):
        table[s, :n] = order[at:at + n]
        at += n
    out = []
    for _ in range(2):
        codes, scales = np.zeros((len(order), hkv, size, d), np.uint8), np.ones((len(order), hkv), np.float32)
        C.append(codes, scales, table, [(s, p) for s, n in enumerate(lens) for p in range(n)],
                 rng.standard_normal((sum(lens), hkv, d)).astype(np.float32))
        out += [codes, scales]
    return table, out


@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (5, 2)])
def test_a_chain_is_the_causal_attention(window, sinks):
    lens, cu = [40, 9], [0, 7, 16]
    table, (ck, sk, cv, sv) = _cache(lens, 16, 2, 64, 0)
    q = np.random.default_rng(1).standard_normal((16, 4, 64))
    named, positions = T.masks([-1, 0, 1, 2, 3, 4, 5] + list(range(-1, 8)), cu, lens, 1)
    got = T.attention(q, ck, sk, cv, sv, table, lens, cu, named, positions, window, sinks, 0.125)
    want = C.attention(q, ck, sk, cv, sv, table, lens, cu, window, sinks, 0.125)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)


def test_a_branch_is_its_path_alone():
    # every row of a tree against a cache that holds its own path and nothing else
    size, base, parents = 16, 21, [-1, 0, 0, 1, -1, 4, 3]
    table, (ck, sk, cv, sv) = _cache([base + 7], size, 1, 64, 2)
    sk[:], sv[:] = 1.0, 0.5                       # (one scale, so that tokens can change places)
    q = np.random.default_rng(3).standard_normal((7, 2, 64))
    named, positions = T.masks(parents, [0, 7], [base + 7], 1)
    o, _, lse, _ = T.attention(q, ck, sk, cv, sv, table, [base + 7], [0, 7], named, positions, 9, 2, 0.2)
    for t in range(7):
        path = np.flatnonzero(named[t])
        k2, v2 = ck.copy(), cv.copy()
        for i, x in enumerate(path):
            for c, of in ((k2, ck), (v2, cv)):
                c[table[0, (base + i) // size], :, (base + i) % size] = of[table[0, (base + x) // size], :, (base + x) % size]
        n = base + len(path)
        w, _, lw, _ = C.attention(q[t:t + 1], k2, sk, v2, sv, table, [n], [0, 1], 9, 2, 0.2)
        assert np.allclose(o[t], w[0], atol=1e-12) and np.allclose(lse[:, t], lw[:, 0], atol=1e-12)


def test_rows_that_see_nothing():
    table, (ck, sk, cv, sv) = _cache([4], 16, 1, 64, 4)
    q = np.ones((4, 1, 64))
    named = np.zeros((4, 64), bool)
    named[1, 1] = True
    o, _, lse, _ = T.attention(q, ck, sk, cv, sv, table, [4], [0, 4], named, np.array([0, 0, -1, 0]), 10, 0, 1.0)
    assert np.isneginf(lse[0, [0, 2, 3]]).all() and np.isfinite(lse[0, 1]) and not o[[0, 2, 3]].any()
    assert np.allclose(o[1, 0], decode_fp8(cv[table[0, 0], 0, 1]) * sv[table[0, 0], 0])


def test_fork_of_a_worked_table():
    table = np.array([[3, 1, 4], [0, 2, -1], [-1, -1, -1]], dtype=np.int32)
    refs = P.counts(table, 6)
    got, lens, counts = P.fork(table, np.array([40, 20, 0]), refs, [0, 0, 1], 16, 2 ** 31 - 1, 0)
    assert got.tolist() == [[3, 1, 4], [3, 1, 4], [0, 2, -1]] and lens.tolist() == [40, 40, 20]
    assert counts.tolist() == [1, 2, 1, 2, 2, 0]
    got, lens, counts = P.fork(table, np.array([30, 20, 0]), refs, None, 16, 2 ** 31 - 1, 0)       # ten tokens taken back
    assert got.tolist() == [[3, 1, -1], [0, 2, -1], [-1, -1, -1]] and counts.tolist() == [1, 1, 1, 1, 0, 0]
    got, _, _ = P.fork(table, np.array([40, 20, 0]), refs, [-1, 1, 5], 16, 2 ** 31 - 1, 0)
    assert got.tolist() == [[-1] * 3, [0, 2, -1], [-1] * 3]
    # window 9 from position 40 on: place 32 and up, and the two sinks of page 0; window 10 sees place 31 too
    assert P.fork(table, np.array([40, 20, 0]), refs, None, 16, 9, 2)[0].tolist()[0] == [3, -1, 4]
    assert P.fork(table, np.array([40, 20, 0]), refs, None, 16, 10, 0)[0].tolist()[0] == [-1, 1, 4]


def test_reserve_of_a_worked_table():
    # rows 0 and 1 share pages 3 and 1 (17 tokens); both write token 17: the second keeps page 1, the first copies it
    table = np.array([[3, 1, -1], [3, 1, -1], [0, -1, -1]], dtype=np.int32)
    refs = P.counts(table, 6)
    got, counts, pairs, missing = P.reserve(table, np.array([18, 18, 17]), refs, [0, 1, 2, 3], 16)
    assert got.tolist() == [[3, 2, -1], [3, 1, -1], [0, 4, -1]] and missing == 0
    assert pairs.tolist() == [[1, 2], [-1, -1], [-1, -1]] and counts.tolist() == [1, 1, 1, 2, 1, 0]
    got, counts, pairs, missing = P.reserve(table, np.array([18, 18, 100]), refs, [0, 1, 2, 85], 16)
    assert missing == 0 and got[2].tolist() == [0, 4, 5]              # places behind the table are left out
    refs[[2, 4, 5]] = 1
    got, counts, pairs, missing = P.reserve(table, np.array([18, 18, 17]), refs, [0, 1, 2, 3], 16)
    assert missing == 2 and np.array_equal(got, table) and np.array_equal(counts, refs) and (pairs == -1).all()


def test_compact_moves_values():
    rng = np.random.default_rng(5)
    lens, size = [50, 33], 16
    table, (codes, scales, _, _) = _cache(lens, size, 2, 64, 6)
    scales *= 2.0 ** rng.integers(-3, 4, scales.shape)

    def values(c, sc, rows, s, places):
        return np.stack([decode_fp8(c[rows[s, p // size], :, p % size]) * sc[rows[s, p // size]][:, None] for p in places])

    keep, cu, first = [20, 21, 30, 47, 49, 5, 9, 32], [0, 5, 8], [18, 3]
    c, sc = codes.copy(), scales.copy()
    P.compact(c, sc, table, table, keep, cu, first)
    for s, n in enumerate((5, 3)):
        old = values(codes, scales, table, s, keep[cu[s]:cu[s + 1]])
        new = values(c, sc, table, s, range(first[s], first[s] + n))
        assert (np.abs(new - old) <= np.maximum(2.0 ** -4 * np.abs(old), 2.0 ** -10 * sc.max())).all()
        kept_old, kept_new = (values(x, y, table, s, range(first[s])) for x, y in ((codes, scales), (c, sc)))
        assert (np.abs(kept_old - kept_new) <= np.maximum(2.0 ** -4 * np.abs(kept_old), 2.0 ** -10 * sc.max())).all()
