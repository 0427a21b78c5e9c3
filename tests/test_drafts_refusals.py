"""Calls of the drafts' entry points that are refused, or are not, at the edges of what their arguments may be (no GPU)."""
import ctypes

from paper_2606_30460_amd import _lib as L
from test_drafts_abi import BAD, FAKE, _append, _compact, _desc, _reserve


def _at(address):
    return ctypes.c_void_p(address)


def test_compaction_whose_lengths_overlap_its_first_places():
    # head 0 writes new_lens[s] while the other heads, and in fresh pages the other pages, still read first
    for dst in (None, FAKE):
        for lens in (8192, 8192 - 8, 8192 + 8):                 # three sequences: twelve bytes
            assert _compact(first=_at(8192), lens=_at(lens), dst=dst) == BAD, lens
            assert "overlap" in L.lib().hsap_last_error().decode()
        for first, lens in ((None, 8192), (8192, None), (8192, 8192 + 12), (8192, 8192 - 12)):
            # (nothing is launched: these have too many heads)
            assert _compact(d=_desc(heads_kv=2 ** 24), first=first and _at(first), lens=lens and _at(lens), dst=dst) == BAD
            assert "too many" in L.lib().hsap_last_error().decode()


def test_an_append_of_nothing_needs_no_positions():
    # (an empty tensor has no address)
    assert _append(cu=FAKE, total=0, positions=None) == L.HSAP_OK
    assert _append(d=_desc(num_seqs=0), total=0, positions=None) == L.HSAP_OK
    assert _append(d=_desc(num_seqs=0), cu=FAKE, total=5, positions=None) == L.HSAP_OK
    assert _append(positions=None) == BAD and _append(cu=FAKE, positions=None) == BAD


def test_reservations_of_more_places_than_their_numbers_hold():
    # places are counted in 32 bits, with a sign
    lib = L.lib()
    for seqs, total in ((2 ** 31 - 1, 5), (2 ** 30, 5), (2 ** 28, 2 ** 20), (2 ** 28 - 2 ** 20, 2 ** 31 - 1)):
        wide = _desc(num_seqs=seqs)
        assert lib.hsap_pages_reserve_workspace(ctypes.byref(wide), total) == -1, (seqs, total)
        assert _reserve(d=wide, total=total) == BAD, (seqs, total)
        assert "too many" in lib.hsap_last_error().decode()
        assert _reserve(d=wide, cu=None, total=seqs) == BAD
    assert lib.hsap_pages_reserve_workspace(ctypes.byref(_desc(num_seqs=2 ** 27)), 2 ** 31 - 1) == 8 * (2 ** 28 + (2 ** 31 - 1) // 16)
