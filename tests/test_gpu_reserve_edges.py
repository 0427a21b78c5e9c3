"""Reservations of pages on the GPU at their edges, against the step-by-step model, exactly."""
import ctypes

import pytest
import torch

from paper_2606_30460_amd import _lib as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages", [1, 3, 64, 20000, 2 ** 31 - 1])
def test_no_sequences(pages):
    """Nothing but `missing` is read or written: no array is needed."""
    desc = L.CacheDesc(num_pages=pages, page_size=16, heads_kv=1, head_dim=64, num_seqs=0, table_width=4)
    missing = torch.full((3,), 9, dtype=torch.int32, device="cuda")
    ws = torch.full((16,), 9, dtype=torch.uint8, device="cuda")
    for cu, total in ((None, 0), (missing.data_ptr(), 5)):
        missing.fill_(9)
        st = L.lib().hsap_pages_reserve(ctypes.byref(desc), None, None, None, cu, total, None, missing.data_ptr() + 4, ws.data_ptr(), 16,
                                        torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == L.HSAP_OK and missing.tolist() == [9, 0, 9] and bool((ws == 9).all())
