"""How an attention call over the paged cache is cut (csrc/cache.h), built for the host."""
import ctypes
import os
import subprocess
import tempfile
from typing import NamedTuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include "%s"
using namespace hsap;
extern "C" void cut(int32_t seqs, int32_t width, int32_t page, int32_t hkv, int32_t d, int32_t hq, int64_t total, int32_t one,
                    int32_t* out) {
  const hsap_cache_desc desc{1, page, hkv, d, seqs, width};
  const CacheCut c = cache_cut(desc, hq, total, one != 0, (int64_t)width * page);
  out[0] = c.rows;
  out[1] = c.splits;
  out[2] = c.once;
}
'''


class Cut(NamedTuple):
    rows: int     # of a workgroup: 16 or 32 (codes in registers), 128 (decoded once through LDS)
    splits: int   # of a row tile's tokens, at most
    once: int     # streaming loads


_lib = None


def cut(seqs, width, page, hkv, d, hq, total, one) -> Cut:
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as tmp:
            src, out = os.path.join(tmp, "cache_h.cpp"), os.path.join(tmp, "cache_h.so")
            with open(src, "w") as f:
                f.write(SOURCE % os.path.join(ROOT, "paper_2606_30460_amd", "csrc", "cache.h"))
            subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                            "-static-libubsan", src, "-o", out], check=True)
            _lib = ctypes.CDLL(out)
    got = (ctypes.c_int32 * 3)()
    _lib.cut(seqs, width, page, hkv, d, hq, ctypes.c_int64(total), int(one), got)
    return Cut(*got)
