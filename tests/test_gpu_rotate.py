"""Rotation by positions of several axes on the GPU: bit for bit against the fp32 model and within half a step of 64 bits;
both ways, types, strides, in place, skipped tokens; and its use in appends to the cache."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from paper_2606_30460_amd import _lib as L
from test_gpu_cache import Pages, _bits, _cos_sin

pytestmark = pytest.mark.gpu


def _rows_of(cs, pair_axis, positions):
    """cos | sin [tokens, rot] of every token's pairs, each from the row of its axis."""
    cs, half = cs.cpu().numpy(), cs.shape[1] // 2
    place = np.clip(positions, 0, len(cs) - 1)[np.asarray(pair_axis)].T          # [tokens, pairs]
    i = np.arange(half)
    return np.concatenate([cs[place, i], cs[place, half + i]], 1)


def _values(shape, g, f32):
    x = torch.randn(shape, generator=g) * torch.exp(torch.randn(shape[0], 1, 1, generator=g))
    return x.cuda() if f32 else x.to(torch.bfloat16).cuda()


def _check(total, hq, hk, d, rot, axes, interleaved=False, inverse=False, types=((0, 0), (0, 0)), strided=False, seed=0, order=None,
           far=False):
    print(total, hq, hk, d, rot, axes, interleaved, inverse, types, strided, flush=True)
    rng = np.random.default_rng(seed)
    pair_axis = {"runs": np.arange(rot // 2) * axes // (rot // 2), "turns": np.arange(rot // 2) % axes,
                 None: rng.integers(0, axes, rot // 2)}[order]
    rows = 300
    positions = rng.integers(-3 if far else 0, rows + (3 if far else 0), (axes, total))
    cs = _cos_sin(rows, rot)
    g = torch.Generator().manual_seed(seed)
    args, expect = [], []
    for heads, (a, b) in zip((hq, hk), types):
        if heads == 0:
            args += [None, None]
            continue
        x = _values((total, heads + (3 if strided else 0), d), g, a)
        x = x[:, 2:2 + heads] if strided else x
        out = torch.full((total, heads + (2 if strided else 0), d), 7.0, dtype=torch.float32 if b else torch.bfloat16, device="cuda")
        view = out[:, 1:1 + heads] if strided else out
        args += [x, view]
        expect.append((x, out, view, b))
    r = L.Rotation(cs, pair_axis, interleaved, axes=axes)
    L.rotate(r, torch.from_numpy(positions.astype(np.int32)).cuda(), *args, inverse=inverse)
    torch.cuda.synchronize()
    table = _rows_of(cs, pair_axis, positions)[:, None]
    if inverse:
        table = np.concatenate([table[..., :rot // 2], -table[..., rot // 2:]], -1)
    live = ((positions >= 0) & (positions < rows)).all(0)
    for x, out, view, b in expect:
        host = x.float().cpu().numpy()
        want = C.rotate(host, table, interleaved, np.float32)
        if not b:
            want = torch.from_numpy(want).to(torch.bfloat16).float().numpy()
        want[~live] = 7.0
        assert np.array_equal(view.float().cpu().numpy(), want)
        wide = C.rotate(host, table, interleaved)       # 64 bits: half a step of the output and the fp32 operations
        tol = (0 if b else 2.0 ** -8) * np.abs(wide) + 2.0 ** -20 * np.abs(host).max(-1, keepdims=True)
        assert (np.abs(want - wide) <= tol)[live].all()
        if strided:
            assert bool((out[:, 0] == 7.0).all()) and bool((out[:, -1] == 7.0).all())


@pytest.mark.parametrize("d,rot", [(64, 16), (64, 64), (128, 48), (128, 128)])
@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("interleaved", [False, True])
def test_axes(d, rot, axes, interleaved):
    for i, order in enumerate(("runs", "turns", None)):
        _check(37, 6, 2, d, rot, axes, interleaved, inverse=i == 1, order=order, seed=axes + i, far=True)


@pytest.mark.parametrize("hq,hk", [(1, 0), (1, 1), (2, 1), (3, 3), (7, 1), (16, 0), (17, 5), (80, 9)])
@pytest.mark.parametrize("d", [64, 128])
def test_heads_and_lengths(d, hq, hk):
    for total in (1, 2, 5, 33, 1000):
        _check(total, hq, hk, d, d // 2, 3, total % 2 == 0, strided=total % 3 == 0, seed=total)


@pytest.mark.parametrize("types", [((0, 0), (1, 0)), ((1, 1), (0, 0)), ((1, 0), (0, 1)), ((1, 1), (1, 1))])
@pytest.mark.parametrize("inverse", [False, True])
def test_types(types, inverse):
    for d, rot, interleaved, strided in ((64, 32, False, True), (128, 128, True, False), (128, 64, False, False), (64, 64, True, True)):
        _check(50, 5, 3, d, rot, 2, interleaved, inverse, types, strided)


def test_nothing():
    r = L.Rotation(_cos_sin(10, 64), [0, 1] * 16)
    q = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    L.rotate(r, torch.empty(2, 0, dtype=torch.int32, device="cuda"), q, q)


def test_in_place_and_the_table_followed():
    for interleaved in (False, True):
        for f32 in (False, True):
            g = torch.Generator().manual_seed(3)
            x, k = _values((77, 6, 128), g, f32), _values((77, 2, 128), g, f32)
            cs = _cos_sin(200, 96)
            r = L.Rotation(cs, np.arange(48) % 3, interleaved)
            p = torch.from_numpy(np.random.default_rng(0).integers(0, 200, (3, 77)).astype(np.int32)).cuda()
            out, ko = torch.empty_like(x), torch.empty_like(k)
            L.rotate(r, p, x, out, k, ko)
            L.rotate(r, p, x, x, k, k)
            torch.cuda.synchronize()
            assert torch.equal(x, out) and torch.equal(k, ko)
            cs[:, 48:] = 0                       # no sines: the cosines alone
            cs[:, :48] = 1
            L.rotate(r, p, out, ko2 := torch.empty_like(out))
            torch.cuda.synchronize()
            assert torch.equal(ko2, out)


def test_non_finite_values_stay_in_their_pairs():
    x = torch.ones(3, 2, 64)
    x[0, 0, 3], x[1, 1, 50], x[2, 0, 60] = float("inf"), float("nan"), float("-inf")
    x = x.to(torch.bfloat16).cuda()
    out = torch.empty_like(x)
    L.rotate(L.Rotation(_cos_sin(10, 32)), torch.zeros(3, dtype=torch.int32, device="cuda") + 5, x, out)
    torch.cuda.synchronize()
    bad = ~torch.isfinite(out.float()).cpu()
    want = torch.zeros_like(bad)
    want[0, 0, [3, 19]] = want[1, 1, 50] = want[2, 0, 60] = True
    assert torch.equal(bad, want)


def test_gradients():
    """Training: q and k turned, then the gradients of the turned rows turned back, against the formula's transpose (a pair's
    products in 64 bits) and against differences of the forward, which is linear, so that they are exact but for rounding."""
    total, hq, hk, d, rot, axes = 19, 4, 2, 64, 48, 3
    g = torch.Generator().manual_seed(5)
    rng = np.random.default_rng(5)
    pair_axis = np.arange(rot // 2) % axes
    positions = rng.integers(0, 100, (axes, total))
    cs = _cos_sin(100, rot)
    r, p = L.Rotation(cs, pair_axis, axes=axes), torch.from_numpy(positions.astype(np.int32)).cuda()
    dq, dk = torch.randn(total, hq, d, generator=g).cuda(), torch.randn(total, hk, d, generator=g).cuda()
    gq, gk = torch.empty_like(dq), torch.empty_like(dk)
    L.rotate(r, p, dq, gq, dk, gk, inverse=True)
    table = _rows_of(cs, pair_axis, positions)
    half = rot // 2
    for up, got in ((dq, gq), (dk, gk)):
        u, got = up.double().cpu().numpy(), got.double().cpu().numpy()
        want = u.copy()
        for t in range(total):
            turn = np.eye(d)
            for i in range(half):
                c, s = float(table[t, i]), float(table[t, half + i])
                turn[i, i], turn[i, i + half], turn[i + half, i], turn[i + half, i + half] = c, -s, s, c
            want[t] = u[t] @ turn
        assert (np.abs(got - want) <= 2.0 ** -20 * np.abs(u).max(-1, keepdims=True)).all()
    # differences: loss = sum(dq * rotate(q)); a unit step of one value
    q = torch.zeros(total, hq, d, device="cuda")
    base, step = torch.empty_like(q), torch.empty_like(q)
    L.rotate(r, p, q, base)
    for _ in range(20):
        at = tuple(int(rng.integers(0, n)) for n in q.shape)
        moved = q.clone()
        moved[at] = 1.0
        L.rotate(r, p, moved, step)
        diff = float(((step - base).double() * dq.double()).sum())
        assert abs(diff - float(gq[at])) <= 2.0 ** -20 * float(dq[at[0], at[1]].abs().max())
    # and back again: turned there and back in fp32, |cos^2 + sin^2 - 1| and four roundings off at most
    L.rotate(r, p, gq, step)
    torch.cuda.synchronize()
    assert bool(((step - dq).abs() <= 2.0 ** -20 * dq.abs().amax(-1, keepdim=True)).all())


def _check_append_at(held, new, size, hkv, d, rot, axes, interleaved=False, hq=0, k_out=False, one=False, seed=0, pad=0, far=False,
                     break_page=None):
    held, new = np.asarray(held), np.asarray(new)
    total = held + new
    p = Pages(np.maximum(total, 0), size, hkv, d, seed).fill(held, seed + 1)
    if break_page is not None:
        p.table[break_page] = 10 ** 6
    n, rows = int(new.sum()), 200
    rng = np.random.default_rng(seed)
    pair_axis = rng.integers(0, axes, rot // 2)
    positions = rng.integers(-10 if far else 0, rows + (10 if far else 0), (axes, n + pad))
    g = torch.Generator().manual_seed(seed)
    fused = (torch.randn(n + pad, hq + 2 * hkv, d, generator=g) * torch.exp(torch.randn(n + pad, 1, 1, generator=g)))
    fused = fused.to(torch.bfloat16).cuda()
    q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    cs = _cos_sin(rows, rot)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    cache = p.device(total)
    q_out = torch.full((n + pad, hq, d), 7.0, dtype=torch.bfloat16, device="cuda") if hq else None
    ko = torch.full((n + pad, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") if k_out else None
    L.cache_append_at(cache, k, v, None if one else torch.from_numpy(cu).cuda(), L.Rotation(cs, pair_axis, interleaved, axes=axes),
                      torch.from_numpy(positions.astype(np.int32)).cuda(), k_out=ko, q=q if hq else None, q_out=q_out)
    torch.cuda.synchronize()
    positions = positions[:, :n]
    seq = np.repeat(np.arange(len(new)), new)
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(held, new)] + [np.zeros(0)]).astype(np.int64)
    live = (pos >= 0) & ((positions >= 0) & (positions < rows)).all(0)
    table = _rows_of(cs, pair_axis, positions)[:, None]
    host = {x: t.float().cpu().numpy()[:n] for x, t in (("q", q), ("k", k), ("v", v))}
    turned = {x: C.rotate(host[x], table, interleaved, np.float32) for x in "qk"}
    turned["v"] = host["v"]
    # (a page begun by a skipped token is begun anew by the others: a page is written by all its tokens at once)
    for x in "kv":
        _append_model(p, x, seq, pos, live, turned[x])
    for x, codes, scale in (("k", cache.k_codes, cache.k_scale), ("v", cache.v_codes, cache.v_scale)):
        assert np.array_equal(_bits(scale), p.scales[x], equal_nan=True), x
        assert np.array_equal(_bits(codes), p.codes[x]), x
    for t, x in ((q_out, "q"), (ko, "k")):
        if t is None:
            continue
        want = torch.from_numpy(turned[x]).to(torch.bfloat16).float().numpy()
        want[~live] = 7.0
        assert np.array_equal(t.float().cpu().numpy()[:n], want), x
        assert bool((t[n:] == 7.0).all())


def _append_model(p, x, seq, pos, live, values):
    """C.append of the tokens that are not skipped.  A page whose first place falls to this call is begun anew, even where that
    token is skipped; places of skipped tokens stay as they were."""
    codes, scales = p.codes[x], p.scales[x]
    places = {}                        # page -> place: written
    for t, (s, a) in enumerate(zip(seq, pos)):
        if 0 <= a < p.table.shape[1] * p.size and 0 <= p.table[s, a // p.size] < len(codes):
            places.setdefault(int(p.table[s, a // p.size]), {})[int(a % p.size)] = bool(live[t])
    old = {page: codes[page].copy() for page in places}
    for page, of in places.items():
        if 0 in of and any(of.values()):
            scales[page] = 0.0         # below every scale, so that it does not count
    C.append(codes, scales, p.table, [(s, int(a)) if ok else (s, -1) for s, a, ok in zip(seq, pos, live)], values)
    for page, of in places.items():
        stay = [i for i in range(p.size) if not of.get(i, 0 not in of)]
        codes[page][:, stay] = old[page][:, stay]


@pytest.mark.parametrize("d,rot,axes,interleaved", [(64, 64, 1, False), (128, 128, 3, True), (128, 96, 3, False), (64, 16, 2, True)])
@pytest.mark.parametrize("size", [16, 32, 64, 128])
def test_append_at_ragged(size, d, rot, axes, interleaved):
    print(size, d, rot, axes, interleaved, flush=True)
    _check_append_at([0, 5, 16, 31, 100, 0, 127], [1, 11, 130, 0, 17, 300, 2], size, 3, d, rot, axes, interleaved, hq=6, k_out=True,
                     seed=size, pad=5)


@pytest.mark.parametrize("size", [16, 128])
def test_append_at_skips_tokens_without_a_row(size):
    for d, interleaved in ((64, False), (128, True)):
        _check_append_at([0, 5, 16, 31, 100, 0], [1, 11, 130, 0, 17, 300], size, 2, d, 64, 4, interleaved, hq=3, k_out=True, seed=size,
                         far=True)
    _check_append_at([3, 30], [20, 30], 16, 2, 64, 32, 2, hq=2, k_out=True, break_page=(1, 2))


@pytest.mark.parametrize("d,rot,axes", [(64, 64, 2), (128, 32, 3)])
@pytest.mark.parametrize("seqs", [1, 7, 70])
def test_append_at_one_token_each(seqs, d, rot, axes):
    held = np.random.default_rng(seqs).integers(1, 60, seqs)
    if seqs > 2:
        held[2] = -1                              # an idle slot: length 0
    print(seqs, d, rot, axes, flush=True)
    _check_append_at(held, np.ones(seqs, int), 64, 2, d, rot, axes, hq=5, k_out=True, one=True, seed=seqs)
    _check_append_at(held, np.ones(seqs, int), 64, 2, d, rot, axes, interleaved=True, hq=5, one=False, seed=seqs + 1)


@pytest.mark.parametrize("interleaved", [False, True])
def test_append_at_its_places_is_the_append(interleaved):
    held, new = np.array([0, 5, 100]), np.array([40, 1, 17])
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
    place = np.concatenate([np.arange(a, a + b) for a, b in zip(held, new)]).astype(np.int32)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(58, h, 128, generator=g).to(torch.bfloat16).cuda() for h in (6, 2, 2))
    cs = _cos_sin(150, 96)
    caches = [Pages(held + new, 32, 2, 128, seed=2).fill(held).device() for _ in range(2)]
    outs = [(torch.empty_like(q), torch.empty_like(k)) for _ in range(2)]
    L.cache_append(caches[0], k, v, cu, cos_sin=cs, interleaved=interleaved, q=q, q_out=outs[0][0], k_out=outs[0][1])
    at = torch.from_numpy(np.stack([place, place, place])).cuda()
    L.cache_append_at(caches[1], k, v, cu, L.Rotation(cs, np.arange(48) % 3, interleaved), at, q=q, q_out=outs[1][0], k_out=outs[1][1])
    torch.cuda.synchronize()
    for a, b in zip(caches[0].tensors + outs[0], caches[1].tensors + outs[1]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_replays_follow_positions_and_lengths():
    held, hkv, d, most = np.array([100, 3, 40]), 2, 128, 50
    p = Pages(held + most, 32, hkv, d, seed=4).fill(held)
    caches = [p.device(held) for _ in range(2)]
    r = L.Rotation(_cos_sin(200, 96), np.arange(48) % 3)
    n = most
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(n, h, d, generator=g).to(torch.bfloat16).cuda() for h in (6, hkv, hkv))
    at, cu = torch.zeros(3, n, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    outs = [[torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k)] for _ in range(2)]

    def step(which):
        L.rotate(r, at, q, outs[which][0], inverse=True)
        L.cache_append_at(caches[which], k, v, cu, r, at, q=q, q_out=outs[which][1], k_out=outs[which][2])

    for which in (0, 1):                           # (all tokens rotated at 0, none appended: what a skipped one keeps)
        step(which)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for turn, new in enumerate(([20, 1, 29], [0, 50, 0], [17, 16, 16])):
        cu.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)))
        at.copy_(torch.randint(-2, 200, at.shape, generator=g, dtype=torch.int32))
        for c in caches:
            c.seq_lens.copy_(torch.from_numpy((held + new).astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        step(1)
        torch.cuda.synchronize()
        for x, y in zip(list(caches[0].tensors) + outs[0], list(caches[1].tensors) + outs[1]):
            same = torch.equal(x.view(torch.uint8), y.view(torch.uint8))
            assert same, turn


def test_refused_arguments():
    cs = _cos_sin(10, 64)
    for bad in (dict(pair_axis=[0] * 31), dict(pair_axis=[4] + [0] * 31), dict(pair_axis=[-1] + [0] * 31), dict(axes=5), dict(axes=0)):
        with pytest.raises(ValueError):
            L.Rotation(cs, **bad)
    r = L.Rotation(cs, [0, 1] * 16)
    q = torch.empty(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    p = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    for at in (p[0], p[:, :3], p.long(), p.cpu(), p.t()):
        with pytest.raises((TypeError, ValueError)):
            L.rotate(r, at, q, q)
    for a, b in ((q.half(), q), (q, q.half()), (q[:, :, ::2], q), (q, q[:2]), (q, q[:, :1]), (q.cpu(), q)):
        with pytest.raises((TypeError, ValueError)):
            L.rotate(r, p, a, b)
    with pytest.raises(ValueError):
        L.rotate(r, p, q, q, k=q)
    with pytest.raises(L.HsapError):
        L.rotate(r, p, torch.empty(4, 2, 32, dtype=torch.bfloat16, device="cuda"), torch.empty(4, 2, 32, dtype=torch.bfloat16, device="cuda"))
