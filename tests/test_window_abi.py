"""Window attention's refusals, before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2606_30460_amd import _lib as L

FAKE = ctypes.c_void_p(4096)     # never dereferenced: the checks fail first
ODD = ctypes.c_void_p(4098)


def _desc(**over):
    s = dict(total_tokens=1001, sp_degree=1, layout=0, shard_id=0, block_m=0, block_n=0, batch=1)
    s.update({k: v for k, v in over.items() if k in s})
    a = dict(heads_q=4, heads_kv=2, head_dim=128, softmax_scale=0.1)
    a.update({k: v for k, v in over.items() if k in a})
    return L.AttnDesc(shard=L.ShardDesc(**s), **a)


def _fwd(d, window=10, sinks=0, q=FAKE, k=FAKE, v=FAKE, cu=FAKE, docs=1, o=FAKE, lse=FAKE):
    return L.lib().hsap_window_attn_fwd(ctypes.byref(d) if d else None, window, sinks, q, k, v, cu, docs, o, lse, None)


def _bwd(d, window=10, sinks=0, q=FAKE, o=FAKE, lse=FAKE, cu=FAKE, docs=1, dq=FAKE, dk=FAKE, wide=0, ws=FAKE, size=1 << 40):
    return L.lib().hsap_window_attn_bwd(ctypes.byref(d) if d else None, window, sinks, q, FAKE, FAKE, FAKE, o, lse, cu, docs,
                                        dq, dk, FAKE, wide, ws, size, None)


@pytest.mark.parametrize("over,code", [
    (dict(head_dim=96), L.HSAP_ERR_UNSUPPORTED),
    (dict(heads_q=3), L.HSAP_ERR_INVALID_ARG),
    (dict(heads_kv=0), L.HSAP_ERR_INVALID_ARG),
    (dict(softmax_scale=0.0), L.HSAP_ERR_INVALID_ARG),
    (dict(softmax_scale=float("inf")), L.HSAP_ERR_INVALID_ARG),
    (dict(total_tokens=0), L.HSAP_ERR_INVALID_ARG),
    (dict(sp_degree=2), L.HSAP_ERR_INVALID_ARG),             # 1001 tokens do not split in two
    (dict(total_tokens=1002, sp_degree=2, layout=1), L.HSAP_ERR_INVALID_ARG),
    (dict(shard_id=1), L.HSAP_ERR_INVALID_ARG),
    (dict(batch=-1), L.HSAP_ERR_INVALID_ARG),
    (dict(heads_q=1 << 20, heads_kv=1 << 20), L.HSAP_ERR_UNSUPPORTED),
])
def test_bad_descriptors(over, code):
    d = _desc(**over)
    assert _fwd(d) == code and _bwd(d) == code
    assert L.lib().hsap_last_error().decode()
    assert L.lib().hsap_window_attn_bwd_workspace(ctypes.byref(d), 10, 0) == -1


def test_bad_arguments():
    d, bad = _desc(), L.HSAP_ERR_INVALID_ARG
    assert _fwd(None) == bad and _bwd(None) == bad
    for call in (_fwd, _bwd):
        assert call(d, window=0) == bad and call(d, window=-5) == bad
        assert call(d, sinks=-1) == bad
        assert call(d, docs=0) == bad
        assert call(d, cu=None) == bad
        assert call(d, q=None) == bad and call(d, q=ODD) == bad
        assert call(d, lse=None) == bad and call(d, o=None) == bad
    assert _fwd(d, o=ODD) == bad
    assert _bwd(d, dq=None) == bad and _bwd(d, dq=ODD) == bad
    assert _bwd(d, dk=ctypes.c_void_p(4104), wide=1) == bad  # fp32 gradients are stored 16 bytes at a time
    assert _bwd(d, ws=None) == bad and _bwd(d, ws=ODD) == bad


def test_backward_workspace_and_sinks():
    lib, d = L.lib(), _desc()
    size = L.window_attn_bwd_workspace(d, 10, 4)
    assert size == (4 * 1001 * 4 + 255) // 256 * 256 + 4 * 2 * 4 * 2 * 128 * 4     # delta, four chunks' partials
    assert L.window_attn_bwd_workspace(d, 1001, 4) == L.window_attn_bwd_workspace(d, 1001, 0)   # nothing beyond the window
    assert _bwd(d, sinks=4, size=size - 1) == L.HSAP_ERR_INVALID_ARG
    assert str(size) in lib.hsap_last_error().decode()
    assert _bwd(d, sinks=129) == L.HSAP_ERR_UNSUPPORTED and "128" in lib.hsap_last_error().decode()
    with pytest.raises(L.HsapError):
        L.window_attn_bwd_workspace(d, 0, 0)
    with pytest.raises(ValueError):
        L.window_attn_bwd_workspace(d, 2 ** 31, 0)


def test_binding_refuses_other_tensors():
    import torch
    d = _desc()
    cpu = torch.zeros(4)
    with pytest.raises(TypeError):
        L.window_attn_fwd(d, 10, 0, cpu, cpu, cpu, cpu, cpu, cpu)
    with pytest.raises(TypeError):
        L.window_attn_bwd(d, 10, 0, cpu, cpu, cpu, cpu, cpu, cpu, cpu, cpu, cpu, cpu, cpu)
