"""Calls at the ends of what the arguments of trees and rotations may be: positions and extents up to 2^31 - 1, lengths below the
drafted tokens, more K heads than Q heads, rows of one tensor turned in place."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from oracle import tree as T
from paper_2606_30460_amd import _lib as L
from test_gpu_cache import _bits, _cos_sin
from test_gpu_rotate import _check as check_rotation
from test_gpu_rotate import _rows_of
from test_gpu_tree import _check, _cu, _masks, _parents

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1

POSITIONS = {
    "far": lambda rng, held: MOST - rng.integers(0, 400, len(held)),
    "near and far": lambda rng, held: np.where(rng.random(len(held)) < 0.5, MOST - rng.integers(0, 3, len(held)),
                                               rng.integers(0, 600, len(held))),
    "none": lambda rng, held: np.where(rng.random(len(held)) < 0.4, -2 ** 31, held + rng.integers(0, 5, len(held))),
}


@pytest.mark.parametrize("what", POSITIONS)
@pytest.mark.parametrize("held,new", [([70, 300, 0], [5, 40, 70]), ([500], [130]), ([33, 2], [3, 1])])
@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 2), (128, 8, 2)])
def test_positions_and_extents_of_any_size(d, hq, hkv, held, new, what):
    rng = np.random.default_rng(len(held) + d)
    words, cu = max(1, -(-max(new) // 64)), _cu(new)
    named = np.zeros((int(cu[-1]), 64 * words), dtype=bool)
    for s, n in enumerate(new):
        named[cu[s]:cu[s + 1], :n] = rng.random((n, n)) < 0.5
    positions = POSITIONS[what](rng, np.repeat(held, new)).astype(np.int64)
    if what == "none":                                       # (a mask names tokens whose positions are not below 0)
        for s, n in enumerate(new):
            named[cu[s]:cu[s + 1], :n] &= positions[cu[s]:cu[s + 1]] >= 0
    for window, sinks in ((MOST, 0), (MOST, MOST), (1, MOST), (1, 0), (MOST - 100, 7), (250, 20), (MOST - 1, 0)):
        print(what, held, new, d, window, sinks, flush=True)
        _check(held, new, 16, hq, hkv, d, window, sinks, seed=1, named=named, positions=positions, words=words)


def test_masks_of_lengths_below_the_drafted_tokens():
    new, lens = [5, 70, 3, 2, 9], np.array([2, 0, -5, MOST, 9])
    rng = np.random.default_rng(0)
    for chain in (False, True):
        parents, cu = _parents(new, rng, chain), _cu(new)
        mask, positions = _masks(parents, cu, lens, 2)
        named, place = T.masks(parents, cu, lens, 2)
        assert np.array_equal(_bits(mask), T.words_of(named)) and np.array_equal(_bits(positions), place)


@pytest.mark.parametrize("hq,hk", [(1, 9), (2, 17), (3, 5)])
@pytest.mark.parametrize("d", [64, 128])
def test_more_k_heads_than_q_heads(d, hq, hk):
    for total in (1, 7, 300):
        check_rotation(total, hq, hk, d, d // 2, 2, total % 2 == 0, strided=total == 7, seed=total)


@pytest.mark.parametrize("total", [1, 2, 333])
@pytest.mark.parametrize("inverse", [False, True])
def test_one_tensor_of_q_k_and_v_in_place(total, inverse):
    hq, hk, d, rot, rows = 5, 2, 64, 48, 100
    rng = np.random.default_rng(total)
    x = torch.randn(total, hq + 2 * hk, d, generator=torch.Generator().manual_seed(total)).to(torch.bfloat16)
    pair_axis, positions, cs = np.arange(rot // 2) % 3, rng.integers(-1, rows, (3, total)), _cos_sin(rows, rot)
    fused = x.cuda()
    q, k = fused[:, :hq], fused[:, hq:hq + hk]
    L.rotate(L.Rotation(cs, pair_axis), torch.from_numpy(positions.astype(np.int32)).cuda(), q, q, k, k, inverse=inverse)
    torch.cuda.synchronize()
    table = _rows_of(cs, pair_axis, positions)[:, None]
    if inverse:
        table = np.concatenate([table[..., :rot // 2], -table[..., rot // 2:]], -1)
    want = x.float().numpy().copy()
    live = (positions >= 0).all(0)
    turned = torch.from_numpy(C.rotate(want[:, :hq + hk], table, False, np.float32)).to(torch.bfloat16).float().numpy()
    want[live, :hq + hk] = turned[live]
    assert np.array_equal(fused.float().cpu().numpy(), want)
