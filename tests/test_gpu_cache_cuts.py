"""Attention over the paged cache in the cuts that large calls take (csrc/cache.h), against the fp64 oracle: streaming loads,
row tiles in few or many splits, 128-row workgroups of single tokens.  A wide table with few pages in use makes a call
large; each case states the cut that its sizes choose, so that a changed rule shows here."""
import numpy as np
import pytest
import torch

from _cache_host import Cut, cut
from paper_2606_30460_amd import _lib as L
from test_gpu_cache import Pages, _attn_only, _check_attn

pytestmark = pytest.mark.gpu

RAGGED = [1, 2, 15, 16, 17, 31, 32, 33, 63, 100, 129, 0, 600]


def _cut(p, hq, total, one):
    return cut(len(p.lens), p.table.shape[1], p.size, p.hkv, p.d, hq, total, one)


@pytest.mark.parametrize("d,width", [(64, 5100), (128, 2600)])
@pytest.mark.parametrize("window,sinks", [(L.MAX_WINDOW, 0), (1, 0), (33, 40), (100, 3), (50, 1000)])
def test_streaming_loads_in_many_splits(window, sinks, d, width):
    print(window, sinks, d, flush=True)
    p = Pages(RAGGED, 16, 2, d, seed=d, width=width).fill(RAGGED)
    assert _cut(p, 8, 13, True) == Cut(16, 39, 1)
    _check_attn(RAGGED, np.ones(13, int), 16, 8, 2, d, window, sinks, seed=d, one=True, pages=p, strided=window == 1)
    assert cut(2, 33000 if d == 64 else 16500, 16, 2, d, 8, 2, True) == Cut(16, 128, 1)
    _check_attn([700, 65], [1, 1], 16, 8, 2, d, window, sinks, seed=d, one=True, width=33000 if d == 64 else 16500)


@pytest.mark.parametrize("d,width", [(64, 700), (128, 360)])
@pytest.mark.parametrize("window,sinks", [(L.MAX_WINDOW, 0), (20, 5)])
def test_streaming_loads_in_few_splits(window, sinks, d, width):
    print(window, sinks, d, flush=True)
    lens = (RAGGED * 2)[:26]
    p = Pages(lens, 16, 8, d, seed=d, width=width).fill(lens)
    assert _cut(p, 16, 26, True) == Cut(16, 4, 1)
    _check_attn(lens, np.ones(26, int), 16, 16, 8, d, window, sinks, seed=d, one=True, pages=p)


@pytest.mark.parametrize("d,width", [(64, 130), (128, 66)])
@pytest.mark.parametrize("window,sinks", [(L.MAX_WINDOW, 0), (9, 2)])
def test_streaming_loads_in_one_part(window, sinks, d, width):
    print(window, sinks, d, flush=True)
    lens = np.random.default_rng(3).integers(0, 50, 132)
    p = Pages(lens, 16, 8, d, seed=d, width=width).fill(lens)
    assert _cut(p, 16, 132, True) == Cut(16, 1, 1)
    _check_attn(lens, np.ones(132, int), 16, 16, 8, d, window, sinks, seed=d, one=True, pages=p)


@pytest.mark.parametrize("d,size,width", [(64, 16, 13200), (128, 16, 6600), (128, 64, 1650)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (20, 0), (21, 3), (40, 17)])
def test_streaming_loads_leave_unseen_places_alone(window, sinks, d, size, width):
    # pages handed back and written by others, NaN codes and scales among them, bad entries in their places
    print(window, sinks, d, size, flush=True)
    lens, hq, one = np.array([300, 77, 3, 129, 160]), 4, np.ones(5, int)
    got = []
    for poison in (False, True):
        p = Pages(lens, size, 2, d, seed=size, width=width).fill(lens)
        assert _cut(p, hq, 5, True).once
        for s, n in enumerate(lens if poison else []):
            j = np.arange(n)
            seen = (n - 1 - j < window) | (j < sinks)
            for page in range(-(-n // size)):
                here = seen[page * size:(page + 1) * size]
                for x in "kv":
                    if not here.any():
                        p.scales[x][p.table[s, page]] = [np.nan, np.inf]
                    p.codes[x][p.table[s, page], :, np.flatnonzero(~here)] = 0xFF
                if not here.any() and s % 2:
                    p.table[s, page] = [2 ** 31 - 1, -5][page % 2]
        got.append(_check_attn(lens, one, size, hq, 2, d, window, sinks, pages=p, one=True) if not poison else
                   _attn_only(p, lens, one, hq, window, sinks, True))
    assert torch.equal(got[0], got[1])


@pytest.mark.parametrize("d,size,width", [(64, 16, 200), (64, 128, 100), (128, 32, 400), (128, 64, 200)])
@pytest.mark.parametrize("window,sinks", [(L.MAX_WINDOW, 0), (1, 0), (70, 3), (300, 100)])
def test_chunks_in_few_splits(window, sinks, d, size, width):
    lens, new = [700, 400], [240, 300]
    print(window, sinks, d, size, flush=True)
    p = Pages(lens, size, 8, d, seed=size, width=width).fill(lens)
    c = _cut(p, 16, sum(new), False)
    assert c.rows == 128 and 2 <= c.splits <= 8
    _check_attn(lens, new, size, 16, 8, d, window, sinks, pages=p, seed=size)


@pytest.mark.parametrize("seqs,splits", [(64, 11), (512, 3)])
def test_single_tokens_of_a_large_group_in_128_rows(seqs, splits):
    # more than 64 query heads to one K/V head
    d, hq = (64, 80) if seqs == 64 else (128, 80)
    lens = np.random.default_rng(5).integers(0, 90 if seqs == 64 else 40, seqs)
    p = Pages(lens, 16, 1, d, seed=seqs, width=260 if d == 64 else 800).fill(lens)
    assert _cut(p, hq, seqs, True) == Cut(128, splits, 0)
    print(seqs, flush=True)
    _check_attn(lens, np.ones(seqs, int), 16, hq, 1, d, window=30, sinks=2, seed=seqs, one=True, pages=p)


@pytest.mark.parametrize("d", [64, 128])
def test_small_row_tiles_in_few_splits(d):
    print(d, flush=True)
    rng = np.random.default_rng(6)
    for most, rows in ((2, 16), (6, 32)):
        lens = rng.integers(0, 200, 20)
        new = np.minimum(rng.integers(0, most + 1, 20), lens)
        p = Pages(lens, 16, 8, d, seed=most, width=100).fill(lens)
        c = _cut(p, 64, int(new.sum()), False)
        assert c.rows == rows and 1 < c.splits <= 8, c
        _check_attn(lens, new, 16, 64, 8, d, window=120, sinks=4, seed=most, pages=p, pad=1)


@pytest.mark.parametrize("one", [True, False])
def test_pages_beyond_32_bits(one):
    # the same sequences in the last pages of a cache of more than 2^32 codes: the bits of a small cache's
    size, hkv, d, hq = 64, 8, 128, 16
    lens, new = np.array([300, 77, 64]), np.ones(3, int) if one else np.array([40, 1, 17])
    p = Pages(lens, size, hkv, d, seed=1).fill(lens - new)
    small = p.device(lens)
    pages, few = 2 ** 32 // (hkv * size * d) + 100, len(p.codes["k"])
    t = {}
    for x in "kv":
        t[x + "_codes"] = torch.zeros((pages, hkv, size, d), dtype=torch.uint8, device="cuda")
        t[x + "_scale"] = torch.zeros((pages, hkv), device="cuda")
        t[x + "_codes"][pages - few:] = getattr(small, x + "_codes")
        t[x + "_scale"][pages - few:] = getattr(small, x + "_scale")
    large = L.KVCache(t["k_codes"], t["v_codes"], t["k_scale"], t["v_scale"], small.page_table + (pages - few), small.seq_lens)
    total = int(new.sum())
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(total, h, d, generator=g).to(torch.bfloat16).cuda() for h in (hq, hkv, hkv))
    cu = None if one else torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    got = []
    for cache in (small, large):
        o = torch.empty_like(q)
        ws = torch.empty(L.cache_attn_workspace(cache, hq, total), dtype=torch.uint8, device="cuda")
        L.cache_append(cache, k, v, cu)
        L.cache_attn(cache, hq, 0.1, q, cu, o, None, ws)
        torch.cuda.synchronize()
        got.append(o)
    assert bool(torch.isfinite(got[0]).all()) and torch.equal(got[0], got[1])
    for x in "kv":
        assert torch.equal(getattr(large, x + "_codes")[pages - few:], getattr(small, x + "_codes"))
        a, b = getattr(large, x + "_scale")[pages - few:], getattr(small, x + "_scale")
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))
        assert not bool(getattr(large, x + "_codes")[:pages - few].any()) and not bool(getattr(large, x + "_scale")[:pages - few].any())
