"""Which pages an attention call over the paged cache looks up (csrc/cache.h, built for the host)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    src = tmp_path_factory.mktemp("cache_steps") / "cache_steps.cpp"
    src.write_text('#include "%s"\nusing namespace hsap;\n'
                   "template <int STEP> int64_t list(int plo, int phi, int cap, int window, int sinks, int32_t* first, int32_t* looked) {\n"
                   "  const Steps<STEP> st = cache_steps<STEP>(plo, phi, cap, window, sinks);\n"
                   "  const int top = phi < cap - 1 ? phi : cap - 1;\n"
                   "  for (int s = 0; s < st.total; ++s) {\n"
                   "    first[s] = st.first(s);\n"
                   "    for (int x = 0; x < STEP / 16; ++x)\n"
                   "      looked[s * (STEP / 16) + x] = st.looked_up(sinks, st.first(s) + 16 * x, top);\n  }\n"
                   "  return st.total;\n}\n"
                   'extern "C" int64_t steps(int step, int plo, int phi, int cap, int window, int sinks, int32_t* f, int32_t* l) {\n'
                   "  return step == 32 ? list<32>(plo, phi, cap, window, sinks, f, l) : list<64>(plo, phi, cap, window, sinks, f, l);\n}\n"
                   % os.path.join(ROOT, "paper_2606_30460_amd", "csrc", "cache.h"))
    out = str(src.with_suffix(".so"))
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-static-libubsan", str(src), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.steps.restype = ctypes.c_int64
    return lib


@pytest.mark.parametrize("step", [32, 64])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (16, 0), (33, 17), (50, 40), (100, 0), (64, 500), (2 ** 31 - 1, 3)])
def test_only_pages_with_a_token_that_some_row_sees(host, step, window, sinks):
    # rows at consecutive positions plo .. phi; pages of sixteen tokens, `cap` tokens in the table
    for cap in (16, 48, 400):
        for plo, phi in ((-5, -1), (-3, 2), (0, 0), (5, 5), (15, 16), (31, 31), (47, 47), (60, 130), (200, 200), (177, 240), (390, 410),
                         (500, 510)):
            first, looked = np.zeros(64, np.int32), np.zeros(256, np.int32)
            total = host.steps(step, plo, phi, cap, window, sinks, *(ctypes.c_void_p(x.ctypes.data) for x in (first, looked)))
            assert total <= 64
            i, j = np.arange(plo, phi + 1)[:, None], np.arange(cap)[None]
            seen = np.flatnonzero(((j <= i) & ((i - j < window) | (j < sinks))).any(0))
            groups = [int(first[s]) + 16 * x for s in range(total) for x in range(step // 16) if looked[s * (step // 16) + x]]
            case = (cap, plo, phi, groups)
            assert set(g // 16 for g in groups) == set(int(t) // 16 for t in seen), case
