"""The paged cache's refusals, before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2606_30460_amd import _lib as L

FAKE = ctypes.c_void_p(4096)     # never dereferenced: the checks fail first
ODD = ctypes.c_void_p(4104)
BAD = L.HSAP_ERR_INVALID_ARG


def _desc(**over):
    a = dict(num_pages=10, page_size=16, heads_kv=2, head_dim=64, num_seqs=3, table_width=4)
    a.update(over)
    return L.CacheDesc(**a)


def _bufs(**over):
    a = dict(k_codes=4096, v_codes=4096, k_scale=4096, v_scale=4096, page_table=4096, seq_lens=4096)
    a.update(over)
    return L.CacheBuffers(**a)


def _append(d=None, c=None, k=FAKE, ks=128, v=FAKE, vs=128, cu=None, total=3, cs=FAKE, rows=100, rot=64, k_out=None, q=None,
            qs=0, hq=0, q_out=None):
    return L.lib().hsap_cache_append(ctypes.byref(d or _desc()), ctypes.byref(c or _bufs()), k, ks, v, vs, cu, total, cs, rows,
                                     rot, 0, k_out, q, qs, hq, q_out, None)


def _attn(d=None, c=None, hq=4, scale=0.1, window=10, sinks=0, q=FAKE, qs=256, cu=None, total=3, o=FAKE, ws=FAKE, size=1 << 40):
    return L.lib().hsap_cache_attn(ctypes.byref(d or _desc()), ctypes.byref(c or _bufs()), hq, scale, window, sinks, q, qs, cu,
                                   total, o, None, ws, size, None)


@pytest.mark.parametrize("over,code", [
    (dict(num_pages=0), BAD), (dict(heads_kv=0), BAD), (dict(num_seqs=-1), BAD), (dict(table_width=0), BAD),
    (dict(page_size=24), L.HSAP_ERR_UNSUPPORTED), (dict(page_size=256), L.HSAP_ERR_UNSUPPORTED),
    (dict(head_dim=96), L.HSAP_ERR_UNSUPPORTED), (dict(table_width=2 ** 28), BAD),
])
def test_bad_caches(over, code):
    assert _append(d=_desc(**over)) == code and _attn(d=_desc(**over)) == code
    assert L.lib().hsap_last_error().decode()


def test_bad_pointers():
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "page_table", "seq_lens"):
        assert _append(c=_bufs(**{name: 0})) == BAD and _attn(c=_bufs(**{name: 0})) == BAD, name
    for name in ("k_codes", "v_codes"):
        assert _append(c=_bufs(**{name: 4104})) == BAD and _attn(c=_bufs(**{name: 4104})) == BAD, name
    lib = L.lib()
    assert lib.hsap_cache_append(None, None, FAKE, 128, FAKE, 128, None, 3, None, 0, 0, 0, None, None, 0, 0, None, None) == BAD


def test_bad_append_arguments():
    assert _append(total=-1) == BAD and _append(total=2) == BAD            # one token each: total_new = num_seqs
    for rot in (-16, 8, 40, 80):
        assert _append(rot=rot) == BAD, rot
    assert _append(cs=None) == BAD and _append(rows=0) == BAD and _append(cs=ODD) == BAD
    assert _append(k=None) == BAD and _append(v=None) == BAD and _append(k=ODD) == BAD
    assert _append(ks=124) == BAD and _append(vs=64) == BAD and _append(ks=132) == BAD
    assert _append(q=FAKE) == BAD and _append(q_out=FAKE) == BAD
    assert _append(q=FAKE, q_out=FAKE, hq=0, qs=256) == BAD and _append(q=FAKE, q_out=FAKE, hq=4, qs=128) == BAD
    assert _append(q=FAKE, q_out=ODD, hq=4, qs=256) == BAD and _append(k_out=ODD) == BAD
    assert _append(d=_desc(num_seqs=0), total=0) == L.HSAP_OK and _append(cu=FAKE, total=0) == L.HSAP_OK   # nothing to do


def test_bad_attention_arguments():
    assert _attn(hq=0) == BAD and _attn(hq=3) == BAD
    assert _attn(scale=0.0) == BAD and _attn(scale=float("nan")) == BAD and _attn(scale=float("inf")) == BAD
    assert _attn(window=0) == BAD and _attn(sinks=-1) == BAD
    assert _attn(total=2) == BAD and _attn(total=-1) == BAD and _attn(cu=FAKE, total=2 ** 30) == BAD
    assert _attn(q=None) == BAD and _attn(q=ODD) == BAD and _attn(o=None) == BAD and _attn(o=ODD) == BAD
    assert _attn(ws=None) == BAD and _attn(ws=ODD) == BAD
    assert _attn(qs=252) == BAD and _attn(qs=192) == BAD
    assert _attn(d=_desc(num_seqs=0), total=0) == L.HSAP_OK and _attn(cu=FAKE, total=0) == L.HSAP_OK


def test_workspace():
    lib = L.lib()
    long = _desc(table_width=1000)
    need = lib.hsap_cache_attn_workspace(ctypes.byref(long), 4, 3, 1)
    assert need > 16
    assert _attn(d=long, size=need - 1) == BAD and str(need) in lib.hsap_last_error().decode()
    for args in ((4, -1, 1), (3, 3, 1), (0, 3, 1)):
        assert lib.hsap_cache_attn_workspace(ctypes.byref(long), *args) == -1
    assert lib.hsap_cache_attn_workspace(None, 4, 3, 1) == -1


def test_binding_refuses_other_tensors():
    import torch
    cpu = torch.zeros(2, 2, 16, 64, dtype=torch.uint8)
    with pytest.raises(TypeError):
        L.KVCache(cpu, cpu, cpu, cpu, cpu, cpu)
