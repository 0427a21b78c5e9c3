"""Refusals of the rotation, tree, compaction and page entry points, before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2606_30460_amd import _lib as L

FAKE = ctypes.c_void_p(4096)     # never dereferenced: the checks fail first
ODD = ctypes.c_void_p(4104)
ODDER = ctypes.c_void_p(4100)
BAD, NONE = L.HSAP_ERR_INVALID_ARG, L.HSAP_ERR_UNSUPPORTED


def _desc(**over):
    a = dict(num_pages=10, page_size=16, heads_kv=2, head_dim=64, num_seqs=3, table_width=4)
    a.update(over)
    return L.CacheDesc(**a)


def _bufs(**over):
    a = dict(k_codes=4096, v_codes=4096, k_scale=4096, v_scale=4096, page_table=4096, seq_lens=4096)
    a.update(over)
    return L.CacheBuffers(**a)


def _rotation(pairs=(0,) * 64, **over):
    a = dict(cos_sin=4096, rows=100, rot_dim=64, interleaved=0, axes=1)
    a.update(over)
    return L.RotationDesc(a["cos_sin"], a["rows"], a["rot_dim"], a["interleaved"], a["axes"], (ctypes.c_uint8 * 64)(*pairs))


def _rows(**over):
    a = dict(src=4096, out=4096, in_stride=256, out_stride=256, heads=4, in_f32=0, out_f32=0)
    a.update(over)
    return L.TokenRows(*a.values())


def _rotate(r=None, d=64, positions=FAKE, total=5, q=None, k=None):
    r, q = r or _rotation(), q or _rows()
    return L.lib().hsap_rotate(ctypes.byref(r), d, positions, total, ctypes.byref(q), None if k is None else ctypes.byref(k), 0, None)


def _append(d=None, c=None, r=None, positions=FAKE, k=FAKE, ks=128, v=FAKE, vs=128, cu=None, total=3, k_out=None, q=None, qs=0, hq=0,
            q_out=None):
    r = r or _rotation()
    return L.lib().hsap_cache_append_at(ctypes.byref(d or _desc()), ctypes.byref(c or _bufs()), k, ks, v, vs, cu, total,
                                        ctypes.byref(r), positions, k_out, q, qs, hq, q_out, None)


def _masks(seqs=3, lens=FAKE, cu=FAKE, total=5, parents=FAKE, words=1, mask=FAKE, positions=FAKE):
    return L.lib().hsap_tree_masks(seqs, lens, cu, total, parents, words, mask, positions, None)


def _attn(d=None, c=None, hq=4, scale=0.1, window=10, sinks=0, q=FAKE, qs=256, cu=FAKE, total=3, mask=FAKE, words=1, positions=FAKE,
          o=FAKE, ws=FAKE, size=1 << 40):
    return L.lib().hsap_cache_tree_attn(ctypes.byref(d or _desc()), ctypes.byref(c or _bufs()), hq, scale, window, sinks, q, qs, cu,
                                        total, mask, words, positions, o, None, ws, size, None)


def _compact(d=None, c=None, keep=FAKE, cu=FAKE, total=3, first=None, dst=None, lens=None):
    return L.lib().hsap_cache_compact(ctypes.byref(d or _desc()), ctypes.byref(c or _bufs()), keep, cu, total, first, dst, lens, None)


def _fork(d=None, table=FAKE, lens=FAKE, refs=FAKE, source=None, window=10, sinks=0):
    return L.lib().hsap_pages_fork(ctypes.byref(d or _desc()), table, lens, refs, source, window, sinks, None)


def _reserve(d=None, table=FAKE, lens=FAKE, refs=FAKE, cu=FAKE, total=5, pairs=FAKE, missing=FAKE, ws=FAKE, size=1 << 40):
    return L.lib().hsap_pages_reserve(ctypes.byref(d or _desc()), table, lens, refs, cu, total, pairs, missing, ws, size, None)


def _copy(d=None, c=None, pairs=FAKE, count=3):
    return L.lib().hsap_cache_copy_pages(ctypes.byref(d or _desc()), ctypes.byref(c or _bufs()), pairs, count, None)


@pytest.mark.parametrize("over,code", [
    (dict(num_pages=0), BAD), (dict(heads_kv=0), BAD), (dict(num_seqs=-1), BAD), (dict(table_width=0), BAD),
    (dict(page_size=24), NONE), (dict(page_size=256), NONE), (dict(head_dim=96), NONE), (dict(table_width=2 ** 28), BAD),
])
def test_bad_caches(over, code):
    for call in (_append, _attn, _compact, _fork, _reserve, _copy):
        assert call(d=_desc(**over)) == code, call.__name__
        assert L.lib().hsap_last_error().decode()


def test_bad_cache_pointers():
    for call in (_append, _attn, _compact, _copy):
        for name in ("k_codes", "v_codes", "k_scale", "v_scale", "page_table", "seq_lens"):
            assert call(c=_bufs(**{name: 0})) == BAD, (call.__name__, name)
        for name in ("k_codes", "v_codes"):
            assert call(c=_bufs(**{name: 4104})) == BAD, (call.__name__, name)


@pytest.mark.parametrize("call", [_rotate, _append])
def test_bad_rotations(call):
    for rot in (-16, 0, 8, 40, 80):
        assert call(r=_rotation(rot_dim=rot)) == BAD, rot
    for axes in (0, 5, -1):
        assert call(r=_rotation(axes=axes)) == BAD, axes
    assert call(r=_rotation(cos_sin=0)) == BAD and call(r=_rotation(cos_sin=4104)) == BAD and call(r=_rotation(rows=0)) == BAD
    assert call(r=_rotation(pairs=[0] * 31 + [2] + [0] * 32, axes=2)) == BAD
    assert call(positions=None) == BAD
    assert L.lib().hsap_last_error().decode()


def test_bad_rotate_arguments():
    assert _rotate(d=96) == NONE and _rotate(total=-1) == BAD and _rotate(total=2 ** 31) == BAD
    for over in (dict(heads=0), dict(src=0), dict(out=0), dict(src=4104), dict(out=4104), dict(in_stride=252), dict(out_stride=252),
                 dict(in_stride=192), dict(out_stride=248)):
        assert _rotate(q=_rows(**over)) == BAD and _rotate(k=_rows(**over)) == BAD, over
    for over in (dict(in_f32=1), dict(out_f32=1), dict(out_stride=264)):         # in place, of two types or strides
        assert _rotate(q=_rows(**over)) == BAD and "in place" in L.lib().hsap_last_error().decode()
    lib = L.lib()
    r, q = _rotation(), _rows()
    assert lib.hsap_rotate(None, 64, FAKE, 5, ctypes.byref(q), None, 0, None) == BAD
    assert lib.hsap_rotate(ctypes.byref(r), 64, FAKE, 5, None, None, 0, None) == BAD
    assert _rotate(total=0, positions=None) == L.HSAP_OK          # nothing to do


def test_bad_append_arguments():
    assert _append(total=-1) == BAD and _append(total=2) == BAD
    assert _append(k=None) == BAD and _append(v=None) == BAD and _append(k=ODD) == BAD
    assert _append(ks=124) == BAD and _append(vs=64) == BAD
    assert _append(q=FAKE) == BAD and _append(q_out=FAKE) == BAD
    assert _append(q=FAKE, q_out=FAKE, hq=0, qs=256) == BAD and _append(q=FAKE, q_out=ODD, hq=4, qs=256) == BAD
    assert _append(k_out=ODD) == BAD and _append(cu=FAKE, total=2 ** 26) == BAD
    assert _append(d=_desc(num_seqs=0), total=0) == L.HSAP_OK and _append(cu=FAKE, total=0) == L.HSAP_OK
    assert L.lib().hsap_cache_append_at(ctypes.byref(_desc()), ctypes.byref(_bufs()), FAKE, 128, FAKE, 128, None, 3, None, FAKE, None,
                                        None, 0, 0, None, None) == BAD


def test_bad_masks():
    assert _masks(seqs=-1) == BAD and _masks(seqs=2 ** 24) == BAD and _masks(total=-1) == BAD and _masks(total=2 ** 31) == BAD
    assert _masks(words=0) == BAD and _masks(words=17) == BAD and _masks(cu=None) == BAD
    for name in ("lens", "parents", "mask", "positions"):
        assert _masks(**{name: None}) == BAD, name
    assert _masks(mask=ODDER) == BAD
    assert _masks(total=0) == L.HSAP_OK and _masks(seqs=0, total=0, cu=None) == L.HSAP_OK


def test_bad_attention_arguments():
    assert _attn(hq=0) == BAD and _attn(hq=3) == BAD
    assert _attn(scale=0.0) == BAD and _attn(scale=float("nan")) == BAD and _attn(scale=float("inf")) == BAD
    assert _attn(window=0) == BAD and _attn(sinks=-1) == BAD
    assert _attn(cu=None, total=2) == BAD and _attn(total=-1) == BAD and _attn(total=2 ** 30) == BAD and _attn(total=2 ** 29 - 1) == BAD
    assert _attn(words=0) == BAD and _attn(words=17) == BAD
    for name in ("q", "o", "ws", "mask", "positions"):
        assert _attn(**{name: None}) == BAD, name
    for name in ("q", "o", "ws"):
        assert _attn(**{name: ODD}) == BAD, name
    assert _attn(mask=ODDER) == BAD
    assert _attn(qs=252) == BAD and _attn(qs=192) == BAD
    assert _attn(d=_desc(num_seqs=0), total=0) == L.HSAP_OK and _attn(total=0) == L.HSAP_OK


def test_attention_workspace():
    lib = L.lib()
    long = _desc(table_width=1000)
    need = lib.hsap_cache_tree_attn_workspace(ctypes.byref(long), 4, 3, 0)
    assert need > 16
    assert _attn(d=long, size=need - 1) == BAD and str(need) in lib.hsap_last_error().decode()
    for args in ((4, -1, 1), (3, 3, 1), (0, 3, 1)):
        assert lib.hsap_cache_tree_attn_workspace(ctypes.byref(long), *args) == -1
    assert lib.hsap_cache_tree_attn_workspace(None, 4, 3, 1) == -1


def test_bad_compactions():
    assert _compact(total=-1) == BAD and _compact(total=2 ** 31) == BAD and _compact(keep=None) == BAD and _compact(cu=None) == BAD
    assert _compact(d=_desc(num_seqs=2 ** 24), total=0) == BAD and _compact(dst=FAKE, total=2 ** 30) == BAD
    assert _compact(d=_desc(num_seqs=0), total=0) == L.HSAP_OK


def test_bad_forks():
    assert _fork(window=0) == BAD and _fork(sinks=-1) == BAD
    for name in ("table", "lens", "refs"):
        assert _fork(**{name: None}) == BAD, name
    assert _fork(d=_desc(num_seqs=16384, table_width=2 ** 27 - 1)) == BAD and "too wide" in L.lib().hsap_last_error().decode()
    assert _fork(d=_desc(num_seqs=16385)) == NONE and _fork(d=_desc(num_seqs=0)) == L.HSAP_OK


def test_bad_reservations():
    assert _reserve(total=-1) == BAD and _reserve(total=2 ** 31) == BAD and _reserve(cu=None) == BAD
    for name in ("table", "lens", "refs", "pairs", "missing", "ws"):
        assert _reserve(**{name: None}) == BAD, name
    assert _reserve(ws=ODD) == BAD
    lib = L.lib()
    need = lib.hsap_pages_reserve_workspace(ctypes.byref(_desc()), 1000)
    assert need >= 8 * (1000 // 16 + 2 * 3)
    assert _reserve(total=1000, size=need - 1) == BAD and str(need) in lib.hsap_last_error().decode()
    assert lib.hsap_pages_reserve_workspace(ctypes.byref(_desc()), -1) == -1
    assert lib.hsap_pages_reserve_workspace(ctypes.byref(_desc(page_size=24)), 5) == -1
    assert lib.hsap_pages_reserve_workspace(None, 5) == -1


def test_bad_copies():
    assert _copy(count=-1) == BAD and _copy(count=2 ** 31) == BAD and _copy(pairs=None) == BAD
    assert _copy(d=_desc(heads_kv=64, page_size=128), count=2 ** 22) == BAD and "too many" in L.lib().hsap_last_error().decode()
    assert _copy(count=0) == L.HSAP_OK


def test_binding_refuses_other_tensors():
    import torch
    cpu = torch.zeros(10, 64)
    with pytest.raises(TypeError):
        L.Rotation(cpu)
