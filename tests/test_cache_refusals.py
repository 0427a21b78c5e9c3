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
