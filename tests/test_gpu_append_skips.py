"""Appends at positions that skip tokens, over several calls: what a page's scale is then, exactly."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from paper_2606_30460_amd import _lib as L
from test_gpu_cache import Pages, _bits, _cos_sin
from test_gpu_rotate import _rows_of

pytestmark = pytest.mark.gpu

HKV, ROWS = 2, 50


def _int32(a):
    return torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda()


def _step(cache, p, lens, new, positions, pair_axis, cs, seed, one):
    """One call on the device and in the model, where a call's tokens that are not skipped are appended and the others are not."""
    n, d = int(np.sum(new)), p.d
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(n, HKV, d, generator=g).to(torch.bfloat16).cuda() for _ in "kv")
    cache.seq_lens.copy_(_int32(lens))
    cu = np.concatenate([[0], np.cumsum(new)])
    L.cache_append_at(cache, k, v, None if one else _int32(cu), L.Rotation(cs, pair_axis, axes=2), _int32(positions))
    torch.cuda.synchronize()
    live = ((positions >= 0) & (positions < ROWS)).all(0)
    seq = np.repeat(np.arange(len(new)), new)
    pos = np.concatenate([np.arange(a - b, a) for a, b in zip(lens, new)])
    at = [(s, int(x)) for s, x, ok in zip(seq, pos, live) if ok]
    turned = C.rotate(k.float().cpu().numpy(), _rows_of(cs, pair_axis, positions)[:, None], False, np.float32)
    for x, values in (("k", turned), ("v", v.float().cpu().numpy())):
        C.append(p.codes[x], p.scales[x], p.table, at, values[live])


def _same(cache, p):
    for x, codes, scale in (("k", cache.k_codes, cache.k_scale), ("v", cache.v_codes, cache.v_scale)):
        assert np.array_equal(_bits(scale), p.scales[x], equal_nan=True), x
        assert np.array_equal(_bits(codes), p.codes[x]), x


def _pages(size, d, former, seed):
    """Sequences whose second page starts with the next token; its scales and codes are its last owner's."""
    p = Pages([2 * size] * 3, size, HKV, d, seed).fill([size] * 3, seed + 1)
    for x in "kv":
        p.codes[x][p.table[:, 1]] = np.random.default_rng(seed).integers(0, 0x7F, (3, HKV, size, d))
        p.scales[x][p.table[:, 1]] = former
    return p, p.device()


@pytest.mark.parametrize("one", [True, False])
@pytest.mark.parametrize("size,d", [(16, 64), (128, 128)])
def test_a_skipped_sequence_stays_as_it_is(size, d, one):
    """Lengths that do not grow and positions of -1: the last place of one sequence, its page's first, holds a token."""
    p, cache = _pages(size, d, 2.0 ** 10, 3)
    cs, pair_axis = _cos_sin(ROWS, d), np.arange(d // 2) % 2
    first = np.array([size + 1] * 3)
    _step(cache, p, first, [1, 1, 1], np.array([[3, 5, 7], [4, 4, 4]]), pair_axis, cs, 0, one)
    _same(cache, p)
    assert (p.scales["v"][p.table[:, 1]] < 1).all()           # begun anew by the token
    _step(cache, p, first, [1, 1, 1], np.array([[-1, ROWS, -1], [4, 4, -1]]), pair_axis, cs, 1, one)
    _same(cache, p)
    _step(cache, p, first + [0, 1, 1], [1, 1, 1], np.array([[-1, 5, 2], [-1, 4, 0]]), pair_axis, cs, 2, one)
    _same(cache, p)


@pytest.mark.parametrize("one", [True, False])
@pytest.mark.parametrize("former", [2.0 ** 10, 2.0 ** -100, float("inf"), float("nan")])
@pytest.mark.parametrize("size,d", [(16, 64), (64, 128)])
def test_a_first_place_left_out_for_good(size, d, former, one):
    p, cache = _pages(size, d, former, 5)
    cs, pair_axis = _cos_sin(ROWS, d), np.arange(d // 2) % 2
    skip, rows = np.full((2, 3), -1), np.array([[3, 5, 7], [1, 0, 2]])
    _step(cache, p, np.full(3, size + 1), [1, 1, 1], skip, pair_axis, cs, 0, one)
    _same(cache, p)                                            # the page's former scale, NaN and infinity too
    for x, scale in (("k", cache.k_scale), ("v", cache.v_scale)):
        scale[_int32(p.table[:, 1]).long()] = 0.0
        p.scales[x][p.table[:, 1]] = 0.0
    _step(cache, p, np.full(3, size + 2), [1, 1, 1], rows, pair_axis, cs, 1, one)
    _same(cache, p)
    for x in "kv":                                             # that of the token alone
        amax = np.abs(p.scales[x][p.table[:, 1]][:, :, None] * 448)
        assert ((amax > 0) & (amax < 2 ** 4)).all()


@pytest.mark.parametrize("former", [2.0 ** 10, 2.0 ** -30])
def test_the_scale_kept_is_that_of_tokens_before(former):
    """Without the caller's 0: a later call takes the page's scale as any append does, whoever made it."""
    p, cache = _pages(32, 64, former, 7)
    cs, pair_axis = _cos_sin(ROWS, 64), np.arange(32) % 2
    _step(cache, p, np.full(3, 35), [3, 3, 3], np.full((2, 9), -1), pair_axis, cs, 0, False)
    _same(cache, p)
    at = np.random.default_rng(0).integers(0, ROWS, (2, 12))
    at[:, 5] = -1
    _step(cache, p, np.full(3, 39), [4, 4, 4], at, pair_axis, cs, 1, False)
    _same(cache, p)
    assert (p.scales["k"][p.table[:, 1]] == former).all() == (former > 1)


def test_an_append_of_nothing():
    """A step without new tokens: empty tensors, which have no address."""
    p = Pages([20] * 3, 16, HKV, 64, 1).fill([20] * 3)
    cache = p.device()
    k = torch.empty(0, HKV, 64, dtype=torch.bfloat16, device="cuda")
    r = L.Rotation(_cos_sin(ROWS, 64), np.arange(32) % 2)
    L.cache_append_at(cache, k, k, _int32([0] * 4), r, torch.empty(2, 0, dtype=torch.int32, device="cuda"), k_out=k, q=k, q_out=k)
    torch.cuda.synchronize()
    _same(cache, p)
