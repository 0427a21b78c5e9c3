"""The window kernels' choices by size (csrc/window.h), built for the host."""
import ctypes
import os
import subprocess
import tempfile
from typing import NamedTuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include "%s"
using namespace hsap;
extern "C" {
int32_t short_row(int32_t x, int32_t g0, int32_t lo, int32_t f, int32_t fe, int32_t last) {
  return short_row_key(x, g0, lo, f, fe, last);
}
void choice(int64_t Ns, int32_t P, int32_t layout, int32_t B, int32_t hq, int32_t hkv, int32_t d, int64_t window, int32_t sinks,
            int32_t* out) {
  Geom g{};
  g.Ns = Ns;
  g.N = B * Ns;
  g.ns = Ns / P;
  g.n = B * g.ns;
  g.m = layout == HSAP_LAYOUT_CONTIGUOUS ? g.ns : g.ns / 2;
  g.P = P;
  g.layout = layout;
  g.B = B;
  hsap_attn_desc a{};
  a.heads_q = hq;
  a.heads_kv = hkv;
  a.head_dim = d;
  const int32_t w = (int32_t)std::min<int64_t>(window, Ns);
  out[0] = window_query_blocks(g, hq, d);
  out[1] = window_row_blocks(window_key_tiles(g, hkv, w), d);
  out[2] = sink_chunks(&a, g, w, sinks);
  out[3] = out[2] ? sink_chunk(&a, g) : 0;
  out[4] = out[2] > kDirectChunks;
  out[5] = head_split(&a, g, w);
}
}
'''


class Choice(NamedTuple):
    query_blocks: int   # 32-row blocks of a workgroup of the forward and of dQ
    key_blocks: int     # of dK/dV
    chunks: int         # sink chunks per segment
    chunk: int          # queries of one
    summed: int         # their partials added up by a launch
    head_split: int     # workgroups that share a key tile's heads


_lib = None


def lib():
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            src, out = os.path.join(d, "window_h.cpp"), os.path.join(d, "window_h.so")
            with open(src, "w") as f:
                f.write(SOURCE % os.path.join(ROOT, "paper_2606_30460_amd", "csrc", "window.h"))
            subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                            "-static-libubsan", src, "-o", out], check=True)
            _lib = ctypes.CDLL(out)
    return _lib


def choice(N, hq, hkv, d, window, sinks, P=1, layout="contiguous", batch=1) -> Choice:
    out = (ctypes.c_int32 * 6)()
    lib().choice(ctypes.c_int64(N), P, 0 if layout == "contiguous" else 1, batch, hq, hkv, d, ctypes.c_int64(window), sinks, out)
    return Choice(*out)
