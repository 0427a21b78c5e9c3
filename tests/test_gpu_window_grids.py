"""Window attention on grids that fill the chip, forward and backward against the fp64 oracle: every shape of workgroup that
the sizes choose (csrc/window.h), the sink pass's longer chunks and their sum.  Each case states what it reaches, so that
a changed rule shows here."""
import numpy as np
import pytest
import torch

import oracle
from _window_host import Choice, choice
from paper_2606_30460_amd import _lib as L
from test_gpu_window import MIX, Problem, _cu

pytestmark = pytest.mark.gpu


def _check_heads(p, kv_heads):
    """p.check for some K/V heads and their query heads; the others' outputs have to be written and finite."""
    out = p.outputs()
    p.forward(out)
    p.backward(out)
    torch.cuda.synchronize()
    grp, end = p.hq // p.hkv, int(p.cu[-1])
    hq = [g * grp + i for g in kv_heads for i in range(grp)]
    q, do = (x[p.pos][:, hq].double().numpy() for x in (p.q, p.do))
    k, v = (x[:, kv_heads].double().numpy() for x in (p.k, p.v))
    ref = oracle.window_attention(q, k, v, p.cu, p.pos, p.window, p.sinks, p.scale, do)
    got = {x: out[x].float().cpu().numpy().astype(np.float64) for x in ("o", "lse", "dq", "dk", "dv")}
    rows, keys = p.pos < end, p.order < end
    for x in got:
        got[x] = got[x].reshape(-1, p.hkv, p.d) if x in ("dk", "dv") else got[x]
        real = got[x][:, rows] if x == "lse" else got[x][keys if x in ("dk", "dv") else rows]
        assert np.isfinite(real).all() and not (real == 7.0).all(-1).any(), x
    for name, real, heads in (("o", rows, hq), ("dq", rows, hq), ("dk", keys, kv_heads), ("dv", keys, kv_heads)):
        r, tol = ref[name], ref[name + "_tol"]
        if name in ("dk", "dv"):
            r, tol = r[p.order], tol[p.order]
        err = np.abs(got[name][:, heads] - r)[real]
        worst = float((err / (tol[real] + 1e-9)).max(initial=0.0))
        assert worst <= 1.0, (name, worst, float(err.max(initial=0.0)))
    assert (np.abs(got["lse"][hq] - ref["lse"])[:, rows] <= ref["lse_tol"][:, rows]).all()


# d, hq, hkv, query and key blocks
GRIDS = [(128, 48, 24, 4, 2), (128, 40, 40, 4, 4), (128, 80, 40, 4, 4), (64, 48, 48, 2, 2), (64, 72, 8, 4, 1), (64, 52, 52, 4, 2),
         (64, 144, 72, 4, 4)]


@pytest.mark.parametrize("d,hq,hkv,qb,kb", GRIDS)
@pytest.mark.parametrize("window,sinks", [(33, 5), (100, 50), (100, 100), (600, 0)])
def test_documents(window, sinks, d, hq, hkv, qb, kb):
    print(window, sinks, d, hq, hkv, flush=True)
    c = choice(600, hq, hkv, d, window, sinks)
    assert (c.query_blocks, c.key_blocks) == (qb, kb)
    assert (c.chunks, c.chunk) == ((3, 256) if sinks else (0, 0))
    Problem(_cu(MIX), 600, window, sinks, d=d, hq=hq, hkv=hkv, seed=window, pad_nan=True, wide_grads=hq == hkv).check()


@pytest.mark.parametrize("N", [1, 33, 127, 129, 159, 257])
@pytest.mark.parametrize("d", [64, 128])
def test_odd_lengths(N, d):
    # key tiles of fewer than 128 rows; heads enough for a grid all the same
    hkv = {64: 272, 128: 144}[d] if N < 256 else {64: 144, 128: 72}[d]
    if N >= 128:
        assert choice(N, hkv, hkv, d, 40, 3).key_blocks == 4
    assert choice(N, hkv, hkv, d, 40, 3).query_blocks == 4
    print(N, d, hkv, flush=True)
    Problem([0, N // 3, N], N, 40, 3, d=d, hq=hkv, hkv=hkv, seed=N).check()


@pytest.mark.parametrize("layout,P,shard,batch,d,hq,hkv,kb", [
    ("zigzag", 2, 1, 1, 128, 48, 48, 4), ("zigzag", 2, 0, 1, 128, 40, 40, 2), ("contiguous", 3, 1, 1, 128, 72, 72, 4),
    ("zigzag", 2, 0, 1, 64, 176, 88, 4), ("contiguous", 1, 0, 3, 64, 64, 32, 4), ("zigzag", 2, 1, 2, 128, 48, 24, 4)])
def test_shards_and_batches(layout, P, shard, batch, d, hq, hkv, kb):
    print(layout, P, shard, batch, d, hq, hkv, flush=True)
    N, window, sinks = 600, 100, 9
    c = choice(N, hq, hkv, d, window, sinks, P, layout, batch)
    assert (c.query_blocks, c.key_blocks, c.chunks > 0) == (4, kb, True)
    Problem(_cu([200, 1, 0, 350, 49] * batch), N, window, sinks, P=P, layout=layout, shard=shard, batch=batch, hq=hq, hkv=hkv,
            d=d, seed=P).check()


@pytest.mark.parametrize("d,hkv,kb", [(128, 40, 2), (128, 72, 4), (64, 80, 2), (64, 136, 4)])
@pytest.mark.parametrize("window,sinks", [(30, 3), (70, 0)])
def test_rows_that_no_query_sees_may_hold_anything(window, sinks, d, hkv, kb):
    print(window, sinks, d, hkv, flush=True)
    P, layout, shard, N, lengths = 3, "zigzag", 1, 720, [100, 1, 560, 59]
    c = choice(N, hkv, hkv, d, window, sinks, P, layout)
    assert c.key_blocks == kb
    p = Problem(_cu(lengths), N, window, sinks, P=P, layout=layout, shard=shard, hq=hkv, hkv=hkv, d=d, seed=P)
    start = np.repeat(np.concatenate([[0], np.cumsum(lengths)[:-1]]), lengths)
    i, j = p.pos[:, None], np.arange(N)[None]
    seen = ((start[i] <= j) & (j <= i) & ((i - j < window) | (j - start[i] < sinks))).any(0)
    finite, out = p.outputs(), p.outputs(fill=-3.0)
    p.forward(finite)
    p.backward(finite)
    unseen = torch.from_numpy(~seen[p.order]).cuda()
    for x in ("k", "v"):
        p.dev[x].view(N, hkv, d)[unseen] = float("nan")
    p.forward(out)
    p.backward(out)
    torch.cuda.synchronize()
    for x in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(finite[x], out[x]), x
    assert not bool(out["dk"].view(N, hkv, d)[unseen].any()) and not bool(out["dv"].view(N, hkv, d)[unseen].any())


@pytest.mark.parametrize("lengths,N,d,hq,hkv,sinks,want", [
    ([700, 1, 499], 1200, 64, 64, 64, 20, Choice(4, 4, 3, 512, 0, 1)),       # chunks of 512
    ([1200], 1200, 128, 64, 64, 60, Choice(4, 4, 3, 512, 0, 1)),
    ([100, 1200], 1300, 64, 102, 102, 128, Choice(4, 4, 2, 1024, 0, 1)),     # and 1024
    ([1024, 276], 1300, 128, 102, 102, 5, Choice(4, 4, 2, 1024, 0, 1)),
    ([30, 2070], 2100, 64, 128, 128, 3, Choice(4, 4, 2, 2048, 0, 1)),        # 2048 and 4096
    ([4200], 4200, 64, 128, 128, 3, Choice(4, 4, 2, 4096, 0, 1)),
    ([300, 2300], 2600, 64, 4, 2, 9, Choice(2, 1, 11, 256, 1, 1)),           # partials summed by a launch
    ([2600], 2600, 64, 24, 24, 40, Choice(4, 4, 11, 256, 1, 1)),
    ([511, 2, 2087], 2600, 128, 24, 24, 100, Choice(4, 4, 11, 256, 1, 1)),
])
def test_sinks_of_long_documents(lengths, N, d, hq, hkv, sinks, want):
    print(lengths, d, hq, hkv, sinks, flush=True)
    c = choice(N, hq, hkv, d, 70, sinks)
    assert c._replace(head_split=1) == want
    _check_heads(Problem(_cu(lengths), N, 70, sinks, hq=hq, hkv=hkv, d=d, seed=sinks), sorted({0, hkv // 2 - 1, hkv - 1}))


def test_same_bits_again_and_replayed():
    # four-block kernels, chunks of 512 and a sum of partials: another stream's call and three replays of a captured one
    for lengths, N, d, hq, hkv in (([700, 1, 499], 1200, 64, 64, 64), ([511, 2, 2087], 2600, 128, 24, 24)):
        print(lengths, flush=True)
        p = Problem(_cu(lengths), N, 70, 5, hq=hq, hkv=hkv, d=d, seed=8)
        assert choice(N, hq, hkv, d, 70, 5).key_blocks == 4
        first, other, cap = p.outputs(), p.outputs(fill=-3.0), p.outputs()
        p.forward(first)
        p.backward(first)
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            p.forward(other)
            p.backward(other)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.forward(cap)
            p.backward(cap)
        names = ("o", "lse", "dq", "dk", "dv")
        for x in names:
            assert torch.equal(first[x], other[x]), x
        for turn in range(3):
            for x in names:
                cap[x].fill_(-turn)
            cap["workspace"].fill_(turn)
            graph.replay()
            torch.cuda.synchronize()
            for x in names:
                assert torch.equal(first[x], cap[x]), (x, turn)
            p.backward(first)                       # eager work between the replays
            torch.cuda.synchronize()


def test_offsets_beyond_32_bits():
    # 70000 rows x 256 heads x 128: q, o and the gradients' last rows lie behind 2^31 elements (and 2^32 bytes)
    n, hq, hkv, d, last, window, sinks = 70000, 256, 2, 128, 90, 40, 3
    assert (n - last) * hq * d > 2 ** 31
    small = Problem([0, last], last, window, sinks, hq=hq, hkv=hkv, d=d, seed=2)
    cu = np.array([0, n - last, n], np.int32)
    p = Problem.__new__(Problem)
    p.__dict__.update(small.__dict__)
    p.desc = L.attn_desc(L.shard_desc(n, 1, "contiguous", 0, 1, 1), hq, hkv, d, small.scale)
    p.n, p.cu_dev = n, torch.from_numpy(cu).cuda()
    for x, t in small.dev.items():
        shape = (1, n, hkv, d) if x in "kv" else (n, hq, d)
        p.dev = dict(p.dev) if p.dev is small.dev else p.dev
        p.dev[x] = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
        p.dev[x].view(n, -1, d)[n - last:] = t.view(last, -1, d)
    out = p.outputs()
    p.forward(out)
    p.backward(out)
    torch.cuda.synchronize()
    ref, _, _ = small.oracle()
    for name in ("o", "dq", "dk", "dv"):
        got = out[name].view(n, -1, d)[n - last:].float().cpu().numpy()
        assert (np.abs(got - ref[name]) <= ref[name + "_tol"] + 1e-9).all(), name
    assert (np.abs(out["lse"][:, n - last:].cpu().numpy() - ref["lse"]) <= ref["lse_tol"]).all()
    assert not bool(out["o"][:n - last].any()) and not bool(out["dq"][:n - last].any())   # zeros elsewhere
