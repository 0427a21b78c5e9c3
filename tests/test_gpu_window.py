"""Window attention with sinks on the GPU against the fp64 oracle, forward and backward, element by element within the
oracle's derived bounds: windows from one token to the whole sequence, sinks, documents of every kind (empty, one
token, longer than a chunk of the sink pass), odd row counts, both layouts, batches, grouped heads, padding rows."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2606_30460_amd import _lib as L

pytestmark = pytest.mark.gpu


def _cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _positions(N, P, layout, shard, batch):
    one = oracle.shard_positions(N, P, layout, shard)
    return np.concatenate([b * N + one for b in range(batch)])


class Problem:
    def __init__(self, cu, N, window, sinks, P=1, layout="contiguous", shard=0, batch=1, hq=2, hkv=1, d=64, seed=0,
                 scale=None, pad_nan=False, wide_grads=False):
        self.cu, self.window, self.sinks, self.hq, self.hkv, self.d = np.asarray(cu, np.int32), window, sinks, hq, hkv, d
        self.scale = scale or 1 / math.sqrt(d)
        g = torch.Generator().manual_seed(seed)
        total = N * batch
        self.q, self.k, self.v, self.do = (torch.randn(total, h, d, generator=g).to(torch.bfloat16) for h in (hq, hkv, hkv, hq))
        if pad_nan:  # what lies behind the last document is never used
            for x in (self.q, self.k, self.v, self.do):
                x[int(self.cu[-1]):] = float("nan")
        self.pos = _positions(N, P, layout, shard, batch)
        self.order = np.concatenate([_positions(N, P, layout, c, batch) for c in range(P)])
        self.desc = L.attn_desc(L.shard_desc(N, P, layout, shard, 1, 1, batch), hq, hkv, d, self.scale)
        self.P, self.n = P, len(self.pos)
        self.dtype = torch.float32 if wide_grads else torch.bfloat16
        self.cu_dev = torch.from_numpy(self.cu).cuda()
        self.dev = {"q": self.q[self.pos].cuda(), "d_o": self.do[self.pos].cuda(),
                    "k": self.k[self.order].view(P, self.n, hkv, d).cuda(), "v": self.v[self.order].view(P, self.n, hkv, d).cuda()}

    def outputs(self, fill=7.0):
        n, hq, hkv, d = self.n, self.hq, self.hkv, self.d

        def full(shape, dtype):
            return torch.full(shape, fill, dtype=dtype, device="cuda")

        out = {"o": full((n, hq, d), torch.bfloat16), "lse": full((hq, n), torch.float32), "dq": full((n, hq, d), torch.bfloat16),
               "dk": full((self.P, n, hkv, d), self.dtype), "dv": full((self.P, n, hkv, d), self.dtype)}
        size = L.window_attn_bwd_workspace(self.desc, self.window, self.sinks)
        out["workspace"] = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN as fp32
        return out

    def forward(self, out, stream=None):
        x = self.dev
        L.window_attn_fwd(self.desc, self.window, self.sinks, x["q"], x["k"], x["v"], self.cu_dev, out["o"], out["lse"], stream)

    def backward(self, out, stream=None):
        x = self.dev
        L.window_attn_bwd(self.desc, self.window, self.sinks, x["q"], x["k"], x["v"], x["d_o"], out["o"], out["lse"],
                          self.cu_dev, out["dq"], out["dk"], out["dv"], out["workspace"], stream)

    def oracle(self):
        end = int(self.cu[-1])
        q, k, v, do = (torch.nan_to_num(x.float()).double().numpy() for x in (self.q, self.k, self.v, self.do))
        ref = oracle.window_attention(q[self.pos], k, v, self.cu, self.pos, self.window, self.sinks, self.scale, do[self.pos])
        return ref, self.pos < end, self.order < end

    def check(self, backward=True):
        out = self.outputs()
        self.forward(out)
        if backward:
            self.backward(out)
        torch.cuda.synchronize()
        ref, rows, keys = self.oracle()
        got = {x: out[x].float().cpu().numpy().astype(np.float64) for x in ("o", "lse", "dq", "dk", "dv")}
        got["dk"], got["dv"] = (got[x].reshape(-1, self.hkv, self.d) for x in ("dk", "dv"))
        names = [("o", rows), ("dq", rows), ("dk", keys), ("dv", keys)] if backward else [("o", rows)]
        for name, real in names:
            r, tol = ref[name], ref[name + "_tol"]
            if name in ("dk", "dv"):
                r, tol = r[self.order], tol[self.order]
            err = np.abs(got[name] - r)[real]
            worst = float((err / (tol[real] + 1e-9)).max(initial=0.0))
            assert worst <= 1.0, (name, worst, float(err.max(initial=0.0)))
            assert (got[name][~real] == 7.0).all(), name + ": padding rows written"
        err = np.abs(got["lse"] - ref["lse"])[:, rows]
        assert (err <= ref["lse_tol"][:, rows]).all(), ("lse", float(err.max()))
        assert (got["lse"][:, ~rows] == 7.0).all()
        return out


MIX = [3, 0, 0, 1, 130, 1, 0, 67, 300, 2, 1, 1, 90]   # 596 tokens


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 5), (31, 0), (64, 4), (100, 33), (128, 128), (257, 3), (596, 0),
                                          (5000, 7), (L.MAX_WINDOW, 0)])
def test_documents_windows_and_sinks(window, sinks, d):
    print("window", window, "sinks", sinks, "d", d, flush=True)
    Problem(_cu(MIX), 596, window, sinks, d=d, hq=4, hkv=2, seed=window).check()


@pytest.mark.parametrize("N", [1, 2, 31, 32, 33, 63, 65, 127, 128, 129, 191, 257])
def test_one_document_of_odd_lengths(N):
    print("N", N, flush=True)
    Problem([0, N], N, 40, 3, d=128, hq=3, hkv=3, seed=N).check()
    Problem([0, N], N, N, 0, d=64, hq=5, hkv=1, seed=N).check()


@pytest.mark.parametrize("layout", ["contiguous", "zigzag"])
@pytest.mark.parametrize("P,shard", [(2, 0), (2, 1), (3, 1), (4, 3)])
def test_shards(layout, P, shard):
    print(layout, P, shard, flush=True)
    N = 12 * 71                                    # 852 tokens: pieces of 426, 213, 284, 142, 106.5 -> odd pieces
    N -= N % (2 * P)
    lengths = [200, 1, 0, 350, 33]
    cu = _cu(lengths + [N - sum(lengths)])
    for window, sinks, d in ((50, 4, 128), (300, 20, 64), (N, 0, 64)):
        Problem(cu, N, window, sinks, P=P, layout=layout, shard=shard, hq=4, hkv=2, d=d, seed=P).check()


@pytest.mark.parametrize("layout,P,shard", [("contiguous", 1, 0), ("contiguous", 2, 1), ("zigzag", 2, 0)])
def test_batches(layout, P, shard):
    N = 300
    cu = _cu([100, 200, 0, 300, 17, 3, 280])       # boundaries at 300 and 600
    for window, sinks in ((33, 2), (128, 0)):
        Problem(cu, N, window, sinks, P=P, layout=layout, shard=shard, batch=3, hq=2, hkv=2, d=64, seed=9).check()


@pytest.mark.parametrize("lengths,N,P,layout,shard", [
    ([2500], 2500, 1, "contiguous", 0),            # three chunks of the sink pass
    ([700, 3000, 300], 4000, 1, "contiguous", 0),  # a document that begins inside a chunk
    ([1024, 2048, 1], 3073, 1, "contiguous", 0),   # documents that begin with a chunk
    ([5, 5995], 6000, 2, "contiguous", 1),         # sinks on the other shard
    ([5, 5995], 6000, 2, "zigzag", 0),             # and chunks in both segments
])
@pytest.mark.parametrize("sinks", [4, 100])
def test_sinks_of_long_documents(lengths, N, P, layout, shard, sinks):
    print(lengths, sinks, flush=True)
    Problem(_cu(lengths), N, 150, sinks, P=P, layout=layout, shard=shard, hq=2, hkv=1, d=128, seed=1).check()


def test_padding_rows_are_not_read_and_not_written():
    for end in (1, 64, 200, 255):
        print("end", end, flush=True)
        Problem([0, end // 2, end], 300, 20, 2, hq=2, hkv=1, d=64, pad_nan=True, seed=end).check()
        Problem([0, end], 300, 300, 0, hq=2, hkv=2, d=128, pad_nan=True, seed=end).check()
    p = Problem([0, 0, 0], 40, 5, 1, pad_nan=True)  # no document at all
    out = p.outputs()
    p.forward(out)
    p.backward(out)
    torch.cuda.synchronize()
    for x in ("o", "lse", "dq", "dk", "dv"):
        assert bool((out[x] == 7.0).all()), x


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout,P,shard", [("contiguous", 4, 2), ("zigzag", 3, 1)])
@pytest.mark.parametrize("window,sinks", [(30, 3), (70, 0)])
def test_rows_that_no_query_sees_may_hold_anything(layout, P, shard, window, sinks, d):
    # the rows of other shards that were never fetched: NaN there gives the bits of finite values there, and gradient 0
    print(layout, P, window, sinks, d, flush=True)
    N, lengths = 240 * P, [100, 1, 240 * P - 160, 59]
    p = Problem(_cu(lengths), N, window, sinks, P=P, layout=layout, shard=shard, hq=4, hkv=2, d=d, seed=P)
    start = np.repeat(np.concatenate([[0], np.cumsum(lengths)[:-1]]), lengths)
    i, j = p.pos[:, None], np.arange(N)[None]
    seen = ((start[i] <= j) & (j <= i) & ((i - j < window) | (j - start[i] < sinks))).any(0)
    assert seen[p.pos].all() and not seen.all()
    finite, out = p.outputs(), p.outputs(fill=-3.0)
    p.forward(finite)
    p.backward(finite)
    unseen = torch.from_numpy(~seen[p.order]).cuda()
    for x in ("k", "v"):
        p.dev[x].view(N, 2, d)[unseen] = float("nan")
    p.forward(out)
    p.backward(out)
    torch.cuda.synchronize()
    for x in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(finite[x], out[x]), x
    assert not bool(out["dk"].view(N, 2, d)[unseen].any()) and not bool(out["dv"].view(N, 2, d)[unseen].any())


def test_many_empty_documents():
    # more boundaries at one position than the kernels' window of boundaries holds
    cu = _cu([10] + [0] * 200 + [30] + [0] * 90 + [1] * 150 + [0] * 70)
    Problem(cu, int(cu[-1]) + 10, 7, 2, hq=2, hkv=1, d=64, pad_nan=True).check()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1), (16, 8), (6, 2), (40, 8)])
def test_head_groups(hq, hkv):
    print(hq, hkv, flush=True)
    Problem(_cu([150, 40]), 190, 60, 2, hq=hq, hkv=hkv, d=64, seed=hq).check()


@pytest.mark.parametrize("d,wide", [(128, False), (64, True)])
def test_heads_of_a_group_in_several_workgroups(d, wide):
    # few key tiles, many heads and a wide window: the heads are dealt out, their parts summed
    for P, layout, shard in ((1, "contiguous", 0), (2, "zigzag", 1)):
        print(P, layout, flush=True)
        p = Problem(_cu([500, 0, 85]), 600, 300, 4, P=P, layout=layout, shard=shard, hq=40, hkv=2, d=d, seed=3, pad_nan=True,
                    wide_grads=wide)
        assert p.outputs()["workspace"].numel() > 2 * P * p.n * 2 * 2 * d * 4
        p.check()


def test_large_scores_and_wide_gradients():
    p = Problem(_cu([170, 30]), 200, 50, 4, hq=2, hkv=1, d=64, scale=2.0, wide_grads=True, seed=4)
    p.check()


def test_full_window_equals_the_planned_forward():
    # the same shard through the planner and the fused forward: both within their bounds of each other
    from paper_2606_30460_amd.shard_attention import ShardAttention
    N, P, r = 1024, 2, 1
    cu = _cu([300, 1, 500, 223])
    p = Problem(cu, N, N, 0, P=P, layout="zigzag", shard=r, hq=4, hkv=2, d=128, seed=6)
    out = p.check(backward=False)
    sa = ShardAttention(cu, N, P, "zigzag", r, 4, 2, 128)
    sa.plan()
    bufs = sa.alloc_forward()
    sa.forward_fused(p.dev["q"], p.dev["k"], p.dev["v"], bufs)
    torch.cuda.synchronize()
    ref, _, _ = p.oracle()
    assert (np.abs((bufs["o"].float() - out["o"].float()).cpu().numpy()) <= 2 * ref["o_tol"]).all()
    assert (np.abs((bufs["lse"] - out["lse"]).cpu().numpy()) <= 2 * ref["lse_tol"]).all()


def test_same_bits_again_on_another_stream_and_replayed():
    p = Problem(_cu([700, 1500]), 2200, 90, 5, hq=4, hkv=2, d=128, seed=8)
    first = p.outputs()
    p.forward(first)
    p.backward(first)
    torch.cuda.synchronize()
    names = ("o", "lse", "dq", "dk", "dv")
    other = p.outputs(fill=-3.0)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        p.forward(other)
        p.backward(other)
    s.synchronize()
    for x in names:
        assert torch.equal(first[x], other[x]), x
    graph, cap = torch.cuda.CUDAGraph(), p.outputs()
    with torch.cuda.graph(graph):
        p.forward(cap)
        p.backward(cap)
    for turn in range(3):
        for x in names:
            cap[x].fill_(-turn)
        cap["workspace"].fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        for x in names:
            assert torch.equal(first[x], cap[x]), (x, turn)
        p.backward(first)                           # eager work between the replays
        torch.cuda.synchronize()
