"""Pins of the cache oracle, and of the kernels' index arithmetic (csrc/cache.h, built for the host) against it."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import oracle
from oracle import cache as C

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rotation_keeps_lengths_and_turns_pairs():
    rng = np.random.default_rng(0)
    x, angle = rng.standard_normal((5, 3, 32)), rng.uniform(0, 6, (5, 1, 8))
    rows = np.concatenate([np.cos(angle), np.sin(angle)], -1)
    for il in (False, True):
        y = C.rotate(x, rows, il)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 16:], x[..., 16:])
        a, b = (x[..., 0:16:2], x[..., 1:16:2]) if il else (x[..., :8], x[..., 8:16])
        want = (a + 1j * b) * np.exp(1j * angle)
        c, d = (y[..., 0:16:2], y[..., 1:16:2]) if il else (y[..., :8], y[..., 8:16])
        assert np.allclose(c + 1j * d, want)


def test_scales_and_codes():
    assert C.scale_of(448) == 1 and C.scale_of(448.0001) == 2 and C.scale_of(1) == 2.0 ** -8 and C.scale_of(0) == 2.0 ** -100
    x = np.random.default_rng(1).standard_normal(1000).astype(np.float32)
    s = C.scale_of(np.abs(x).max())
    back = oracle.decode_fp8(C.encode(x / np.float32(s))) * s
    assert (np.abs(back - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * s).all()


def test_append_token_by_token_is_near_one_append():
    rng = np.random.default_rng(2)
    x = (rng.standard_normal((40, 2, 16)) * np.exp(rng.uniform(-3, 3, (40, 1, 1)))).astype(np.float32)
    table = np.array([[2, 0, 1]], dtype=np.int32)
    one = [np.zeros((3, 2, 16, 16), np.uint8), np.zeros((3, 2), np.float32)]
    C.append(*one, table, [(0, p) for p in range(40)], x)
    many = [np.full((3, 2, 16, 16), 0x7F, np.uint8), np.full((3, 2), np.nan, np.float32)]
    for p in range(40):
        C.append(*many, table, [(0, p)], x[p:p + 1])
    assert np.array_equal(one[1], many[1])
    a, b = (oracle.decode_fp8(c) * s.astype(np.float64)[:, :, None, None] for c, s in (one, many))
    # re-encoding loses only what falls among the subnormals: half their step, 2^-10 of the scale, each time
    assert (np.abs(a - b)[[2, 0]] <= 2.0 ** -9 * one[1][[2, 0]][:, :, None, None] + 2.0 ** -4 * np.abs(a)[[2, 0]]).all()


def test_attention_against_the_packed_oracle():
    rng = np.random.default_rng(3)
    k, v, q = (rng.standard_normal((37, h, 16)).astype(np.float32) for h in (2, 2, 4))
    table = np.array([[4, 1, 3]], dtype=np.int32)
    ck, cv, sk, sv = np.zeros((5, 2, 16, 16), np.uint8), np.zeros((5, 2, 16, 16), np.uint8), np.zeros((5, 2), np.float32), \
        np.zeros((5, 2), np.float32)
    C.append(ck, sk, table, [(0, p) for p in range(37)], k)
    C.append(cv, sv, table, [(0, p) for p in range(37)], v)

    def held(c, s):
        x = oracle.decode_fp8(c[table[0]]) * s[table[0]].astype(np.float64)[:, :, None, None]
        return x.transpose(0, 2, 1, 3).reshape(48, 2, 16)[:37]

    for window, sinks in ((100, 0), (5, 3)):
        o, _, lse, _ = C.attention(q[30:].astype(np.float64), ck, sk, cv, sv, table, [37], [0, 7], window, sinks, 0.25)
        ref = oracle.window_attention(q[30:], held(ck, sk), held(cv, sv), [0, 37], np.arange(30, 37), window, sinks, 0.25)
        assert np.allclose(o, ref["o"], atol=1e-12) and np.allclose(lse, ref["lse"], atol=1e-12)


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    src = tmp_path_factory.mktemp("cache_h") / "cache_h.cpp"
    src.write_text('#include "%s"\nusing namespace hsap;\nextern "C" {\n'
                   "int32_t page_of(const int32_t* r, int32_t w, int32_t n, int32_t s, int32_t p) { return cache_page(r, w, n, s, p); }\n"
                   "int64_t row_of(int64_t p, int32_t hs, int32_t h, int32_t s, int32_t t, int32_t d) { return cache_row(p, hs, h, s, t, d); }\n"
                   "int64_t base_of(int64_t c, int64_t n, int64_t d, int64_t a, int64_t s) { return item_base(c, n, d, a, s); }\n"
                   "int exp_of(uint32_t b) { return scale_exponent(b); }\n}\n"
                   % os.path.join(ROOT, "paper_2606_30460_amd", "csrc", "cache.h"))
    out = str(src.with_suffix(".so"))
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-static-libubsan", str(src), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.row_of.restype = lib.base_of.restype = ctypes.c_int64
    lib.row_of.argtypes = [ctypes.c_int64] + [ctypes.c_int32] * 5
    lib.base_of.argtypes = [ctypes.c_int64] * 5
    return lib


def test_pages_of_positions_and_bad_entries(host):
    row = (ctypes.c_int32 * 4)(3, -1, 9, 0)
    for p in range(-3, 80):
        want = -1
        if 0 <= p < 64:
            want = {0: 3, 1: -1, 2: -1, 3: 0}[p // 16]
        assert host.page_of(row, 4, 9, 16, p) == want, p
    assert host.page_of(row, 4, 9, 16, 2 ** 31 - 1) == -1
    assert host.row_of(2 ** 20, 8, 3, 128, 5, 128) == ((2 ** 20 * 8 + 3) * 128 + 5) * 128     # beyond 32 bits


def test_ragged_work_items_cover_every_page_and_row(host):
    rng = np.random.default_rng(4)
    for _ in range(300):
        seqs, ps = int(rng.integers(1, 9)), int(rng.choice([16, 32]))
        new = rng.choice([0, 1, 2, 15, 16, 17, 33, 100], seqs)
        held = rng.integers(0, 70, seqs)
        cu = np.concatenate([[0], np.cumsum(new)])
        base = [host.base_of(int(c), 1, ps, 2, s) for s, c in enumerate(cu)]
        for s in range(seqs):       # pages that the new tokens reach fit the items up to the next base
            pages = (held[s] + new[s] - 1) // ps - held[s] // ps + 1 if new[s] else 0
            assert base[s] + pages <= base[s + 1]
        group, rows = int(rng.integers(1, 9)), int(rng.choice([16, 32, 64]))
        base = [host.base_of(int(c), group, rows, 1, s) for s, c in enumerate(cu)]
        for s in range(seqs):
            assert base[s] + -(-int(new[s]) * group // rows) <= base[s + 1]


def test_scale_exponents(host):
    rng = np.random.default_rng(5)
    x = np.concatenate([np.exp(rng.uniform(-90, 88, 3000)), 448.0 * 2.0 ** np.arange(-130, 119),
                        np.nextafter((448.0 * 2.0 ** np.arange(-110, 119)).astype(np.float32), np.float32(np.inf)), [0.0]])
    x = x.astype(np.float32)
    for bits, a in zip(x.view(np.uint32), x):
        assert 2.0 ** host.exp_of(ctypes.c_uint32(int(bits))) == C.scale_of(float(a)), a
