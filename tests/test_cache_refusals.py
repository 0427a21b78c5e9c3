"""Calls on the paged cache that are refused for their size, before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2606_30460_amd import _lib as L

FAKE = ctypes.c_void_p(4096)     # never dereferenced: the checks fail first


def _desc(**over):
    a = dict(num_pages=10, page_size=16, heads_kv=2, head_dim=64, num_seqs=3, table_width=4)
    a.update(over)
    return L.CacheDesc(**a)


def _bufs():
    return L.CacheBuffers(4096, 4096, 4096, 4096, 4096, 4096)


@pytest.mark.parametrize("total,heads_q", [(2 ** 26, 0), (2 ** 20, 4096)])
def test_appends_of_more_threads_than_a_launch_has(total, heads_q):
    # 2^32 threads and more: by the pages' workgroups, by Q's
    q = FAKE if heads_q else None
    st = L.lib().hsap_cache_append(ctypes.byref(_desc()), ctypes.byref(_bufs()), FAKE, 128, FAKE, 128, FAKE, total, None, 0, 0, 0,
                                   None, q, heads_q * 64, heads_q, q, None)
    assert st == L.HSAP_ERR_INVALID_ARG and "too many" in L.lib().hsap_last_error().decode()


def test_attention_of_more_threads_than_a_launch_has():
    total, heads_q = 2 ** 29 - 1, 4
    st = L.lib().hsap_cache_attn(ctypes.byref(_desc()), ctypes.byref(_bufs()), heads_q, 0.1, 10, 0, FAKE, 256, FAKE, total, FAKE,
                                 None, FAKE, 2 ** 60, None)
    assert st == L.HSAP_ERR_INVALID_ARG and "too many" in L.lib().hsap_last_error().decode()


def test_workspace_of_what_the_call_refuses():
    lib, heads_q, total = L.lib(), 4, 3
    assert lib.hsap_cache_attn_workspace(ctypes.byref(_desc()), heads_q, total, 1) >= 0
    for over in (dict(page_size=24), dict(page_size=256), dict(table_width=2 ** 28), dict(head_dim=96), dict(table_width=0)):
        d = _desc(**over)
        st = lib.hsap_cache_attn(ctypes.byref(d), ctypes.byref(_bufs()), heads_q, 0.1, 10, 0, FAKE, 256, None, total, FAKE, None, FAKE,
                                 2 ** 60, None)
        assert st != L.HSAP_OK, over
        assert lib.hsap_cache_attn_workspace(ctypes.byref(d), heads_q, total, 1) == -1 and lib.hsap_last_error().decode(), over
    assert lib.hsap_cache_attn_workspace(ctypes.byref(_desc()), heads_q, 2 ** 29, 0) == -1     # total_q x heads_q beyond 32 bits
