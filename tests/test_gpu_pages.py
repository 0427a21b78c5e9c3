"""Pages of the cache on the GPU: forks, reservations, copies and compactions against the step-by-step models, exactly; lists and
tables of every kind, replays, offsets beyond 32 bits."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from oracle import pages as P
from paper_2606_30460_amd import _lib as L
from test_gpu_cache import Pages, _bits

pytestmark = pytest.mark.gpu


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(dtype))).cuda()


def _cu(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def _cache(table, lens, pages, size=16, hkv=1, d=64):
    shape = (pages, hkv, size, d)
    return L.KVCache(torch.zeros(shape, dtype=torch.uint8, device="cuda"), torch.zeros(shape, dtype=torch.uint8, device="cuda"),
                     torch.ones(shape[:2], device="cuda"), torch.ones(shape[:2], device="cuda"), _dev(table), _dev(lens))


def _table(lens, width, pages, size, rng, share=0.0):
    """Rows with pages for their tokens, some shared with an earlier row's same places."""
    table, free = np.full((len(lens), width), -1, dtype=np.int32), list(rng.permutation(pages))
    for s, n in enumerate(lens):
        like = int(rng.integers(0, s)) if s and rng.random() < share else None
        for c in range(min(width, -(-max(0, int(n)) // size))):
            take = table[like, c] if like is not None else -1
            table[s, c] = take if take >= 0 else free.pop()
    return table


def _check_fork(lens, width, size, source, window=L.MAX_WINDOW, sinks=0, seed=0, pages=None, share=0.3, other=False):
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    pages = pages or sum(-(-max(0, int(n)) // size) for n in lens) + 5
    table = _table(lens, width, pages, size, rng, share)
    refs = P.counts(table, pages)
    refs[rng.integers(0, pages)] += 3                        # a page that the caller keeps in another way
    cache, r = _cache(table, lens * 0 if other else lens, pages, size), _dev(refs)
    committed = _dev(lens) if other else None
    L.pages_fork(cache, r, None if source is None else _dev(source), seq_lens=committed, window=window, sinks=sinks)
    torch.cuda.synchronize()
    want, want_lens, want_refs = P.fork(table, lens, refs, source, size, window, sinks)
    assert np.array_equal(_bits(cache.page_table), want)
    assert np.array_equal(_bits(committed if other else cache.seq_lens), want_lens)
    if other:
        assert not bool(cache.seq_lens.any())
    assert np.array_equal(_bits(r), want_refs)


@pytest.mark.parametrize("size", [16, 32, 64, 128])
def test_fork(size):
    lens = [0, 1, size - 1, size, size + 1, 300, 5 * size, 777, 40, 12]
    rng = np.random.default_rng(size)
    for source in (None, np.arange(10), np.full(10, 7), rng.permutation(10), rng.integers(-2, 13, 10), np.full(10, -1),
                   np.array([2 ** 31 - 1, -2 ** 31] * 5), np.roll(np.arange(10), 1)):
        _check_fork(lens, 60, size, source, seed=size, other=source is not None and source[0] == 0)
        _check_fork(lens, 60, size, source, window=100, sinks=3, seed=size + 1)
        _check_fork(lens, 60, size, source, window=1, seed=size + 2)


def test_fork_of_tables_of_every_shape():
    rng = np.random.default_rng(0)
    for rows, width in ((1, 1), (1, 1000), (300, 33), (512, 32), (4000, 1), (600, 40), (2000, 7), (8192, 1), (16384, 1)):
        lens = rng.integers(0, 16 * width + 1, rows)
        print(rows, width, flush=True)
        _check_fork(lens, width, 16, rng.integers(-1, rows, rows), seed=rows)
        _check_fork(lens, width, 16, None, window=50, seed=rows)


def test_fork_gives_back_what_lies_behind_the_lengths():
    table = np.array([[3, 1, 4], [0, 2, -1]])
    cache, refs = _cache(table, [17, 0], 6), _dev([1, 1, 1, 1, 1, 0])
    L.pages_fork(cache, refs)
    torch.cuda.synchronize()
    assert cache.page_table.tolist() == [[3, 1, -1], [-1, -1, -1]] and refs.tolist() == [0, 1, 0, 1, 0, 0]
    cache.page_table = _dev([[3, 1, 77], [-5, 2, -1]])          # entries that are no pages are none
    L.pages_fork(cache, refs, _dev([1, 0]))
    torch.cuda.synchronize()
    assert cache.page_table.tolist() == [[-1, -1, -1], [3, 1, -1]] and cache.seq_lens.tolist() == [0, 17]


def _check_reserve(lens, new, width, size, seed=0, spare=0, share=0.5, one=False, pad=0, shift=0):
    """Rows that hold lens - new tokens, some of them shared, get pages for all."""
    rng = np.random.default_rng(seed)
    lens, new = np.asarray(lens), np.asarray(new)
    held = np.maximum(lens - new, 0)
    need = sum(-(-max(0, int(n)) // size) for n in lens) + len(lens)
    pages = sum(-(-int(n) // size) for n in held) + need + 3
    table = _table(held, width, pages, size, rng, share)
    # the same page at the same place means the same tokens: shared rows hold as many tokens as the shorter
    refs = P.counts(table, pages)
    if spare is not None:                                   # so many free pages alone
        free = np.flatnonzero(refs == 0)
        refs[rng.permutation(free)[spare:] if spare else free[:0]] = 1
    cu = _cu(new)
    cache, r = _cache(table, lens, pages, size), _dev(refs)
    pairs, missing = torch.full((len(lens), 2), 9, dtype=torch.int32, device="cuda"), torch.full((1,), 9, dtype=torch.int32, device="cuda")
    total = int(cu[-1]) + pad
    ws = torch.full((L.pages_reserve_workspace(cache, total),), 0xFF, dtype=torch.uint8, device="cuda")
    L.pages_reserve(cache, r, None if one else _dev(cu), total, pairs, missing, ws)
    torch.cuda.synchronize()
    want, want_refs, want_pairs, short = P.reserve(table, lens, refs, cu, size)
    assert int(missing) == short, (int(missing), short)
    assert np.array_equal(_bits(cache.page_table), want) and np.array_equal(_bits(r), want_refs)
    assert np.array_equal(_bits(pairs), want_pairs)
    return short


@pytest.mark.parametrize("size", [16, 32, 64, 128])
def test_reserve(size):
    lens = np.array([1, 0, size - 1, size, size + 1, 300, 5 * size, 777, 40, 12, 3 * size + 1])
    rng = np.random.default_rng(size)
    for seed in range(6):
        new = np.minimum(lens, rng.choice([0, 1, 1, 2, 17, size, 300], len(lens)))
        print(size, seed, new.tolist(), flush=True)
        _check_reserve(lens, new, 60, size, seed=seed, pad=seed % 2)
        _check_reserve(lens, new, 60, size, seed=seed, share=1.0)
        _check_reserve(lens, new, 3, size, seed=seed)         # places behind the table
    _check_reserve(lens, np.ones(len(lens), int), 60, size, one=True, share=0.8)
    _check_reserve([5, 3], [9, 3], 4, size)                   # more new tokens than tokens


def test_reserve_with_too_few_pages():
    seen = set()
    for seed in range(8):
        lens = np.random.default_rng(seed).integers(1, 400, 20)
        new = np.minimum(lens, np.random.default_rng(seed + 50).integers(0, 60, 20))
        for spare in (1, 5, 12, 40, 200):
            seen.add(_check_reserve(lens, new, 30, 16, seed=seed, spare=spare, share=0.7) > 0)
    assert seen == {False, True}


def test_reserve_among_many_pages_and_rows():
    rng = np.random.default_rng(1)
    for rows, most in ((3000, 40), (50, 3000), (1, 16 * 5000), (1500, 900)):
        lens = rng.integers(1, most + 1, rows)
        new = np.minimum(lens, rng.integers(0, most // 2 + 2, rows))
        print(rows, most, flush=True)
        _check_reserve(lens, new, -(-most // 16), 16, seed=rows, share=0.3)


def test_reserve_shared_by_all_and_by_some():
    # four rows share one partial page: all write (the last keeps it), three write, and a page begun anew is not copied
    for writers in ([1, 1, 1, 1], [1, 0, 1, 1], [0, 0, 1, 0]):
        for held in (20, 32):
            table = np.array([[5, 2, -1]] * 4)
            refs = P.counts(table, 12)
            new = np.array(writers)
            lens = held + new
            cache, r = _cache(table, lens, 12), _dev(refs)
            pairs, missing = torch.empty(4, 2, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
            ws = torch.empty(L.pages_reserve_workspace(cache, 4), dtype=torch.uint8, device="cuda")
            L.pages_reserve(cache, r, _dev(_cu(new)), 4, pairs, missing, ws)
            torch.cuda.synchronize()
            want, want_refs, want_pairs, _ = P.reserve(table, lens, refs, _cu(new), 16)
            assert np.array_equal(_bits(cache.page_table), want) and np.array_equal(_bits(r), want_refs)
            assert np.array_equal(_bits(pairs), want_pairs)
    # tokens taken back into shared pages: every one that is written again is left to the others
    table = np.array([[1, 2, 3], [1, 2, 3]])
    refs = P.counts(table, 9)
    cache, r = _cache(table, [48, 48], 9), _dev(refs)
    L.pages_reserve(cache, r, _dev([0, 40, 40]), 40, pairs := torch.empty(2, 2, dtype=torch.int32, device="cuda"),
                    torch.empty(1, dtype=torch.int32, device="cuda"),
                    torch.empty(L.pages_reserve_workspace(cache, 40), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert cache.page_table.tolist() == [[0, 4, 5], [1, 2, 3]] and pairs.tolist() == [[1, 0], [-1, -1]]
    assert r.tolist() == [1, 1, 1, 1, 1, 1, 0, 0, 0]


@pytest.mark.parametrize("rows", [3, 1500])
def test_reserve_of_a_page_twice_in_a_row(rows):
    # one page at two places of the same sequence, both written: the last one keeps it
    table = np.full((rows, 4), -1)
    table[:, :3] = np.arange(rows)[:, None] * 2 + np.array([0, 1, 1])
    refs = P.counts(table, 2 * rows + 9)
    refs[-9:-7] = 1
    lens, new = np.full(rows, 20), np.zeros(rows, int)
    lens[[0, rows - 1]], new[[0, rows - 1]] = 40, 20                # places 20 .. 39: the second page, partly, and the third
    cache, r = _cache(table, lens, len(refs)), _dev(refs)
    pairs, missing = torch.empty(rows, 2, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(L.pages_reserve_workspace(cache, 40), dtype=torch.uint8, device="cuda")
    L.pages_reserve(cache, r, _dev(_cu(new)), 40, pairs, missing, ws)
    torch.cuda.synchronize()
    want, want_refs, want_pairs, short = P.reserve(table, lens, refs, _cu(new), 16)
    assert int(missing) == short == 0 and np.array_equal(_bits(pairs), want_pairs)
    got = _bits(cache.page_table)
    assert np.array_equal(got, want) and np.array_equal(_bits(r), want_refs) and got[0, 1] != got[0, 2] == 1


@pytest.mark.parametrize("size,hkv,d", [(16, 1, 64), (32, 3, 128), (128, 8, 128), (64, 5, 64), (128, 9, 128)])
def test_copy_pages(size, hkv, d):
    print(size, hkv, d, flush=True)
    p = Pages([20 * size], size, hkv, d, spare=8).fill([20 * size])
    cache = p.device()
    free = sorted(set(range(28)) - set(p.table[0].tolist()))
    pairs = [[p.table[0, 3], free[0]], [-1, -1], [p.table[0, 3], free[2]], [5, 5], [28, 2], [3, 10 ** 6], [-1, 4], [p.table[0, 7], free[7]],
             [2 ** 31 - 1, -2 ** 31]]
    L.cache_copy_pages(cache, _dev(pairs))
    torch.cuda.synchronize()
    for a, b in ((pairs[0]), (pairs[2]), (pairs[7])):
        for x in "kv":
            p.codes[x][b], p.scales[x][b] = p.codes[x][a], p.scales[x][a]
    for x, c, sc in (("k", cache.k_codes, cache.k_scale), ("v", cache.v_codes, cache.v_scale)):
        assert np.array_equal(_bits(c), p.codes[x]) and np.array_equal(_bits(sc), p.scales[x], equal_nan=True)
    L.cache_copy_pages(cache, torch.empty(0, 2, dtype=torch.int32, device="cuda"))


def _check_compact(lens, kept, first, size, hkv, d, fresh=False, seed=0, spread=1.0, pad=0, scale=False, width=None, edit=None,
                   aliased=False):
    """kept: places per sequence."""
    p = Pages(lens, size, hkv, d, seed, spare=3 + (sum(-(-len(k) // size) + 1 for k in kept) if fresh else 0), width=width)
    p.fill(lens, seed + 1, spread=spread)
    if scale:
        for x in "kv":
            p.scales[x] *= np.random.default_rng(seed).uniform(0.3, 3.0, p.scales[x].shape).astype(np.float32)
    target = p.table.copy()
    if fresh:
        free = [x for x in range(len(p.codes["k"])) if x not in set(p.table.ravel().tolist())]
        for s, k in enumerate(kept):
            f = 0 if first is None else max(0, first[s])
            for c in range(f // size, min(target.shape[1], (f + len(k) - 1) // size + 1 if len(k) else 0)):
                target[s, c] = free.pop()
                if c * size < f:               # a page that holds the tokens before: some, of a scale of its own
                    for x in "kv":
                        p.codes[x][target[s, c]] = p.codes[x][p.table[s, c]]
                        p.scales[x][target[s, c]] = p.scales[x][p.table[s, c]]
    if edit:
        edit(p, target)
    cu = _cu([len(k) for k in kept])
    keep = np.concatenate([np.asarray(k, dtype=np.int64) for k in kept] + [np.full(pad, 10 ** 6)]).astype(np.int32)
    cache = p.device(lens)
    out = cache.seq_lens if aliased else torch.full((len(lens),), 9, dtype=torch.int32, device="cuda")
    L.cache_compact(cache, _dev(keep), _dev(cu), first=None if first is None else _dev(first), dst_table=_dev(target) if fresh else None,
                    new_lens=out)
    torch.cuda.synchronize()
    f = np.zeros(len(lens), int) if first is None else np.maximum(first, 0)
    for x, codes, scales in (("k", cache.k_codes, cache.k_scale), ("v", cache.v_codes, cache.v_scale)):
        P.compact(p.codes[x], p.scales[x], p.table, target, keep, cu, f)
        assert np.array_equal(_bits(scales), p.scales[x], equal_nan=True), x
        assert np.array_equal(_bits(codes), p.codes[x]), x
    assert out.tolist() == [int(a) + len(k) for a, k in zip(f, kept)]


def _some(lens, first, share, rng):
    return [np.sort(rng.permutation(np.arange(a, n))[:int(round(share * (n - a)))]) for a, n in zip(first, lens)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [16, 32, 64, 128])
@pytest.mark.parametrize("fresh", [False, True])
def test_compact(fresh, size, d):
    lens = [1, 20, size, 2 * size + 1, 300, 5 * size, 77, 40]
    rng = np.random.default_rng(size)
    for i, share in enumerate((0.0, 0.1, 0.5, 0.9, 1.0)):
        print(fresh, size, d, share, flush=True)
        first = [0, 3, size // 2, size, 250, 0, 77, 17]
        _check_compact(lens, _some(lens, first, share, rng), first, size, 3, d, fresh, seed=i, spread=1.5, pad=i)
        _check_compact(lens, _some(lens, [0] * 8, share, rng), None, size, 2, d, fresh, seed=i, aliased=i == 2)


def test_compact_of_accepted_tokens():
    # the last page's tokens, one to all of them, over its border
    for base in (0, 5, 15, 16, 31):
        for n in (1, 2, 17, 40):
            for k in ([0], [n - 1], [0, n - 1] if n > 1 else [0], list(range(n))):
                _check_compact([base + n], [[base + x for x in k]], [base], 16, 2, 64, seed=base)


def test_compact_raises_and_lowers_scales():
    # spread over many binades: subnormal codes, pages whose scale rises by the moved tokens, zeros from pages of large scale
    for seed in range(6):
        lens = [200, 130]
        first = [20, 0]
        _check_compact(lens, _some(lens, first, 0.4, np.random.default_rng(seed)), first, 16, 2, 64, seed % 2 == 1, seed=seed, spread=6.0)

    def zeros(p, target):
        for x in "kv":
            p.scales[x][p.table[0, 2]] = 2.0 ** 120
            p.codes[x][p.table[0, 2]] = 0
            p.codes[x][p.table[0, 3], :, 1] = 0x7E              # 448 of a scale of its own
            p.codes[x][p.table[0, 3], :, 5] = 0xFF              # NaN: stays, counts for nothing
            p.codes[x][p.table[0, 4], :, 2] = 0x80              # -0
            p.scales[x][p.table[0, 4]] = 2.0 ** -100

    _check_compact([80], [list(range(32, 48))], [0], 16, 1, 64, edit=zeros)
    _check_compact([80], [[33, 40, 49, 66, 70]], [0], 16, 1, 64, edit=zeros)
    _check_compact([80], [[66, 67]], [0], 16, 1, 64, edit=zeros)
    _check_compact([80], [[33, 40, 49, 66]], [3], 16, 1, 64, True, edit=zeros)


def test_compact_of_other_scales():
    lens, first = [100, 200], [10, 0]
    for fresh in (False, True):
        p = _some(lens, first, 0.5, np.random.default_rng(1))
        _check_compact(lens, p, first, 32, 2, 128, fresh, scale=True, seed=4)


def test_compact_of_places_without_a_page():
    def edit(p, target):
        p.table[0, 4] = 10 ** 6                                  # tokens of no page: zeros
        target[0, 4] = p.table[0, 4] if (p.table == target).sum() > 5 else target[0, 4]
    for fresh in (False, True):
        _check_compact([200], [[3, 5, 64, 66, 70, 100, 150, 4000, 2 ** 31 - 1]], [0], 16, 2, 64, fresh, edit=edit)

    def no_target(p, target):
        target[0, 1] = -1                                        # nowhere to go: dropped
    _check_compact([200], [list(range(10, 60))], [0], 16, 2, 64, True, edit=no_target)
    _check_compact([64], [[5, 60]], [63], 16, 1, 64, True, width=4)      # the second behind the table


def test_compact_of_idle_sequences():
    _check_compact([0, 30, 0], [[], [], []], [0, 30, -4], 16, 1, 64)
    _check_compact([40, 30], [[5, 6], []], [-7, 30], 16, 1, 64, aliased=True)
    cache = _cache(np.zeros((1, 1)), [3], 1)
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    L.cache_compact(cache, empty, _dev([0, 0]))


def test_replays():
    """A captured step of branching: fork, reserve, copy, against the same calls made eagerly."""
    rows, size, pages = 6, 16, 80
    rng = np.random.default_rng(3)
    lens = np.array([20, 0, 0, 35, 0, 0])
    table = _table(lens, 8, pages, size, rng)
    new, total = _dev([1, 2, 3, 4, 5, 1]), 16
    cu = _dev(_cu([1, 2, 3, 4, 5, 1]))
    states = []
    for _ in range(2):
        c = _cache(table, lens, pages, size, 2, 64)
        c.k_codes.copy_(torch.randint(0, 120, c.k_codes.shape, generator=torch.Generator().manual_seed(1), dtype=torch.uint8))
        states.append(dict(c=c, refs=_dev(P.counts(table, pages)), lens=_dev(lens), source=_dev([0, 0, 0, 3, 3, 3]),
                           pairs=torch.empty(rows, 2, dtype=torch.int32, device="cuda"),
                           missing=torch.empty(1, dtype=torch.int32, device="cuda"),
                           ws=torch.empty(L.pages_reserve_workspace(c, total), dtype=torch.uint8, device="cuda")))

    def step(s):
        L.pages_fork(s["c"], s["refs"], s["source"], seq_lens=s["lens"])
        torch.add(s["lens"], new, out=s["c"].seq_lens)
        L.pages_reserve(s["c"], s["refs"], cu, total, s["pairs"], s["missing"], s["ws"])
        L.cache_copy_pages(s["c"], s["pairs"])

    for s in states:
        step(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(states[0])
    for turn, source in enumerate(([0, 0, 0, 3, 3, 3], [2, 2, 2, 5, 5, 5], [0, 1, 2, 2, 1, 0], [-1, 1, 4, 3, 3, -1])):
        for s in states:
            s["source"].copy_(_dev(source))
            if turn % 2:
                s["lens"].add_(new)
        graph.replay()
        torch.cuda.synchronize()
        step(states[1])
        torch.cuda.synchronize()
        a, b = states
        for x in ("refs", "lens", "pairs", "missing"):
            assert torch.equal(a[x], b[x]), (turn, x)
        for x, y in zip(a["c"].tensors, b["c"].tensors):
            assert torch.equal(x, y), turn
        assert int(a["missing"]) == 0
        assert np.array_equal(_bits(a["refs"]), P.counts(_bits(a["c"].page_table), pages))


def test_offsets_beyond_32_bits():
    """Copies and moves in a cache of more than 2^32 bytes per tensor."""
    hkv, size, d = 8, 128, 128
    page = hkv * size * d
    pages = 2 ** 32 // page + 40
    codes = [torch.zeros((pages, hkv, size, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones((pages, hkv), device="cuda") for _ in range(2)]
    last = pages - 1
    table = torch.tensor([[last - 3, last - 2], [last - 1, 5]], dtype=torch.int32, device="cuda")
    cache = L.KVCache(*codes, *scales, table, torch.tensor([200, 200], dtype=torch.int32, device="cuda"))
    g = torch.Generator().manual_seed(0)
    for c in codes:
        for x in (last - 3, last - 2, last - 1, 5):
            c[x] = torch.randint(0, 120, (hkv, size, d), generator=g, dtype=torch.uint8).cuda()
    L.cache_copy_pages(cache, _dev([[last - 1, last], [last - 3, 7], [5, last - 4]]))
    torch.cuda.synchronize()
    for c in codes:
        assert torch.equal(c[last], c[last - 1]) and torch.equal(c[7], c[last - 3]) and torch.equal(c[last - 4], c[5])
    want = [torch.cat([c[last - 2][:, 3:5], c[last - 2][:, 60:61]], 1).clone() for c in codes]
    keep, cu = _dev([131, 132, 188]), _dev([0, 3, 3])
    L.cache_compact(cache, keep, cu, first=_dev([100, 0]))
    torch.cuda.synchronize()
    for c, w in zip(codes, want):
        assert torch.equal(c[last - 3][:, 100:103], w)


def test_refused_arguments():
    cache = _cache(np.zeros((2, 3)), [1, 1], 9)
    refs = torch.zeros(9, dtype=torch.int32, device="cuda")
    two, pairs = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    for call in (lambda: L.pages_fork(cache, refs[:8]), lambda: L.pages_fork(cache, refs.long()), lambda: L.pages_fork(cache, refs, two[:1]),
                 lambda: L.pages_fork(cache, refs.cpu()), lambda: L.pages_fork(cache, refs, seq_lens=two[:1]),
                 lambda: L.cache_copy_pages(cache, two), lambda: L.cache_copy_pages(cache, pairs.long()),
                 lambda: L.cache_compact(cache, two, two), lambda: L.cache_compact(cache, two, _dev([0, 1, 2]), first=two[:1]),
                 lambda: L.cache_compact(cache, two, _dev([0, 1, 2]), dst_table=two),
                 lambda: L.cache_compact(cache, two, _dev([0, 1, 2]), new_lens=two.long()),
                 lambda: L.pages_reserve(cache, refs, None, 2, pairs[:1], two[:1], torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            call()
    with pytest.raises(L.HsapError):
        L.pages_fork(cache, refs, window=0)
    with pytest.raises(L.HsapError):
        L.pages_reserve(cache, refs, None, 3, pairs, two[:1], torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(L.HsapError):
        L.pages_reserve(cache, refs, None, 2, pairs, two[:1], torch.empty(0, dtype=torch.uint8, device="cuda"))
