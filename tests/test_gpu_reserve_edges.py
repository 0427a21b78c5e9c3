"""Reservations of pages on the GPU at their edges, against the step-by-step model, exactly."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import pages as P
from paper_2606_30460_amd import _lib as L
from test_gpu_pages import _bits, _cache, _cu, _dev, _table

pytestmark = pytest.mark.gpu

FEW = 1024      # places (a bound of them: total / size + 2 a sequence) that are held in registers; more take several passes
STRETCH = 16 * 1024     # pages that one look at refs takes in


@pytest.mark.parametrize("pages", [1, 3, 64, 20000, 2 ** 31 - 1])
def test_no_sequences(pages):
    """Nothing but `missing` is read or written: no array is needed."""
    desc = L.CacheDesc(num_pages=pages, page_size=16, heads_kv=1, head_dim=64, num_seqs=0, table_width=4)
    missing = torch.full((3,), 9, dtype=torch.int32, device="cuda")
    ws = torch.full((16,), 9, dtype=torch.uint8, device="cuda")
    for cu, total in ((None, 0), (missing.data_ptr(), 5)):
        missing.fill_(9)
        st = L.lib().hsap_pages_reserve(ctypes.byref(desc), None, None, None, cu, total, None, missing.data_ptr() + 4, ws.data_ptr(), 16,
                                        torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == L.HSAP_OK and missing.tolist() == [9, 0, 9] and bool((ws == 9).all())


class Rows:
    """A table of rows that hold `lens` - `new` tokens, and `pages` pages of which `free` (numbers) are free."""

    def __init__(self, lens, new, width, pages, share, seed, free=None, size=16):
        self.lens, self.new, self.size = np.asarray(lens), np.asarray(new), size
        rng = np.random.default_rng(seed)
        held = np.maximum(self.lens - self.new, 0)
        self.table = _table(held, width, pages, size, rng, share)
        used = P.counts(self.table, pages)
        self.refs = used.copy()
        if free is not None:
            self.refs[used == 0] = 1                        # pages that the caller keeps in another way
            self.refs[free] = used[free]
        self.cu = _cu(self.new)

    @property
    def places(self):
        return int(self.cu[-1]) // self.size + 2 * len(self.lens)

    def check(self, shift=0):
        """refs at 4 * shift bytes behind an aligned address."""
        n, total = len(self.lens), int(self.cu[-1])
        cache = _cache(self.table, self.lens, len(self.refs), self.size)
        refs = torch.full((len(self.refs) + 8,), 1, dtype=torch.int32, device="cuda")
        refs[:] = 0                                         # (free ones on both sides, which are none of the cache's)
        r = refs[shift:shift + len(self.refs)]
        r.copy_(_dev(self.refs))
        pairs, missing = torch.full((n, 2), 9, dtype=torch.int32, device="cuda"), torch.full((1,), 9, dtype=torch.int32, device="cuda")
        ws = torch.full((L.pages_reserve_workspace(cache, total),), 0xFF, dtype=torch.uint8, device="cuda")
        L.pages_reserve(cache, r, _dev(self.cu), total, pairs, missing, ws)
        torch.cuda.synchronize()
        want, want_refs, want_pairs, short = P.reserve(self.table, self.lens, self.refs, self.cu, self.size)
        assert int(missing) == short, (int(missing), short)
        assert np.array_equal(_bits(cache.page_table), want) and np.array_equal(_bits(r), want_refs)
        assert np.array_equal(_bits(pairs), want_pairs)
        assert not bool(refs[:shift].any()) and not bool(refs[shift + len(self.refs):].any())
        return short


def _shared_by_writers(lens, new, table, size):
    """Entries whose page is shared, by rows that all write it and by rows that do not all."""
    count, writers = {}, {}
    for s, row in enumerate(table):
        for c, p in enumerate(row):
            if p < 0:
                continue
            count[p] = count.get(p, 0) + 1
            if new[s] and max(0, lens[s] - new[s]) // size <= c <= (lens[s] - 1) // size:
                writers[p] = writers.get(p, 0) + 1
    shared = [p for p, n in count.items() if n > 1 and p in writers]
    return sum(writers[p] == count[p] for p in shared), sum(writers[p] < count[p] for p in shared)


@pytest.mark.parametrize("rows", [700, 3000])
def test_many_places_with_too_few_pages(rows):
    """Everything is put back: pages kept by the last of their writers among them."""
    seen = set()
    for seed in range(3):
        rng = np.random.default_rng(seed)
        lens = rng.integers(1, 120, rows)
        new = np.minimum(lens, rng.choice([0, 1, 1, 3, 20, 40], rows))
        x = Rows(lens, new, 8, 10 * rows, 0.7, seed)
        assert x.places > FEW
        need = len(np.flatnonzero(x.refs == 0)) - np.count_nonzero(P.reserve(x.table, lens, x.refs, x.cu, 16)[1] == 0)
        every = np.flatnonzero(x.refs == 0)
        all_write, some_write = _shared_by_writers(lens, new, x.table, 16)
        assert all_write > 5 and some_write > 5
        for spare in (0, 1, need // 2, need - 1, need, need + 1):
            y = Rows(lens, new, 8, 10 * rows, 0.7, seed, free=rng.permutation(every)[:spare])
            short = y.check(shift=spare % 4)
            assert short == max(0, need - spare), (seed, spare)
            seen.add(short > 0)
    assert seen == {False, True}


def test_many_places_shared_by_their_writers_alone():
    # every page is shared by two rows; both write it, or one of them, and the pages that are free are one too few or enough
    rows, size = 1200, 16
    for spare in (rows // 2 - 1, rows // 2):
        table = np.full((rows, 3), -1)
        table[:, 0] = np.arange(rows) // 2
        x = Rows(np.full(rows, 9), np.ones(rows, int), 3, 2 * rows, 0.0, 0)
        x.table, x.refs = table, P.counts(table, 2 * rows)
        x.refs[rows // 2 + spare:] = 1
        assert x.check() == rows // 2 - spare
    for spare in (rows // 4 - 1, rows // 4):                # (the second of every other pair alone writes)
        new = np.tile([0, 1, 0, 0], rows // 4)
        x = Rows(8 + new, new, 3, 2 * rows, 0.0, 0)
        x.table, x.refs = table, P.counts(table, 2 * rows)
        x.refs[rows // 2 + spare:] = 1
        assert x.check() == rows // 4 - spare


@pytest.mark.parametrize("pages", [STRETCH + 1, STRETCH + 2003, 2 * STRETCH + 3001, 3 * STRETCH + 2507])
@pytest.mark.parametrize("rows", [40, 1100])
def test_free_pages_far_behind(rows, pages):
    """The free pages lie behind the first stretch, in the last one, or on both sides of a border; few places and many."""
    rng = np.random.default_rng(pages)
    lens = rng.integers(1, 90, rows)
    new = np.minimum(lens, rng.integers(0, 40, rows))
    base = Rows(lens, new, 8, pages, 0.5, 1)
    assert (base.places > FEW) == (rows > 40)
    every = np.flatnonzero(base.refs == 0)
    need = len(every) - np.count_nonzero(P.reserve(base.table, lens, base.refs, base.cu, 16)[1] == 0)
    last = every[every >= (pages - 1) // STRETCH * STRETCH]
    border = every[(every >= STRETCH - need // 2)]
    for what, free in (("last", last), ("last, just enough", last[:need]), ("too few", last[:need - 1]), ("none", last[:0]),
                       ("border", border[:need]), ("border, too few", border[:need - 1]), ("behind the first", every[every >= STRETCH])):
        x = Rows(lens, new, 8, pages, 0.5, 1, free=free)
        print(rows, pages, what, len(free), need, flush=True)
        assert x.check() == max(0, need - len(free))


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("pages", [1, 2, 3, 5, 301, 1024])
def test_counts_at_any_address(pages, shift):
    rows = min(pages, 30)
    lens = np.random.default_rng(pages).integers(1, 17, rows) if pages > 5 else np.full(rows, 16)
    new = np.ones(rows, int)
    new[: rows // 2] = lens[: rows // 2]
    x = Rows(lens, new, 4, pages, 0.4, 2)
    x.check(shift)
    x = Rows(lens, lens, 4, pages, 0.0, 2, free=np.arange(pages)[::2])
    x.check(shift)


@pytest.mark.parametrize("rows", [8191, 8192, 8193, 9500])
def test_rows_by_the_thousand(rows):
    """The sequences are searched in LDS up to 8192 of them, else in memory."""
    rng = np.random.default_rng(rows)
    lens = rng.integers(0, 60, rows)
    new = np.minimum(lens, rng.choice([0, 0, 1, 2, 30], rows))
    x = Rows(lens, new, 4, 6 * rows, 0.4, 3)
    assert x.check() == 0
    y = Rows(lens, new, 4, 6 * rows, 0.4, 3, free=np.flatnonzero(x.refs == 0)[:50])
    assert y.check() > 0


def test_replays_of_many_places():
    rows, width, pages = 900, 6, 9000
    rng = np.random.default_rng(1)
    lens = rng.integers(1, 80, rows)
    states = []
    for k in range(2):
        x = Rows(lens, np.minimum(lens, 3), width, pages, 0.6, 5)
        c = _cache(x.table, lens, pages)
        states.append(dict(c=c, refs=_dev(x.refs), cu=_dev(x.cu), pairs=torch.empty(rows, 2, dtype=torch.int32, device="cuda"),
                           missing=torch.empty(1, dtype=torch.int32, device="cuda"),
                           ws=torch.empty(L.pages_reserve_workspace(c, 3 * rows), dtype=torch.uint8, device="cuda")))

    def step(s):
        L.pages_reserve(s["c"], s["refs"], s["cu"], 3 * rows, s["pairs"], s["missing"], s["ws"])

    for s in states:
        step(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(states[0])
    for turn in range(4):
        new = np.minimum(lens, rng.integers(0, 4, rows))
        x = Rows(lens, new, width, pages, 0.6, 10 + turn)
        refs = x.refs.copy()
        if turn % 2:
            refs[np.flatnonzero(refs == 0)[20:]] = 1        # too few
        for s in states:
            s["c"].page_table.copy_(_dev(x.table))
            s["refs"].copy_(_dev(refs))
            s["cu"].copy_(_dev(x.cu))
        graph.replay()
        torch.cuda.synchronize()
        step(states[1])
        torch.cuda.synchronize()
        a, b = states
        want, want_refs, want_pairs, short = P.reserve(x.table, lens, refs, x.cu, 16)
        for s in states:
            assert int(s["missing"]) == short and (short > 0) == bool(turn % 2)
            assert np.array_equal(_bits(s["c"].page_table), want) and np.array_equal(_bits(s["refs"]), want_refs)
            assert np.array_equal(_bits(s["pairs"]), want_pairs)
