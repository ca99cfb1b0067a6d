"""The paged cache's C ABI on the host: bad shapes and null handles are rejected
before touching the GPU."""
import ctypes

import pytest

from paper_2608_02438_amd import xpress as X


def _shape(**kw):
    s = dict(n_heads=32, n_kv=8, head_dim=128, page_size=16, n_pages=1000, dtype=X.XP_BF16)
    s.update(kw)
    return X._KvShape(**s)


@pytest.mark.parametrize("change,status", [
    (dict(head_dim=96), X.XP_EUNSUPPORTED),
    (dict(head_dim=0), X.XP_EINVAL),
    (dict(n_kv=3), X.XP_EUNSUPPORTED),             # 32 heads not a multiple of 3
    (dict(n_kv=0), X.XP_EINVAL),
    (dict(n_heads=130, n_kv=2), X.XP_EUNSUPPORTED),   # a group of 65
    (dict(page_size=8), X.XP_EUNSUPPORTED),
    (dict(page_size=48), X.XP_EUNSUPPORTED),
    (dict(page_size=512), X.XP_EUNSUPPORTED),
    (dict(n_pages=0), X.XP_EINVAL),
    (dict(n_pages=1 << 27), X.XP_EUNSUPPORTED),    # slots past 31 bits
    (dict(dtype=X.XP_F32), X.XP_EINVAL),
    (dict(dtype=7), X.XP_EINVAL),
])
def test_create_rejects_shapes(change, status):
    L = X.load_library()
    h = ctypes.c_void_p(0)
    assert L.xp_kv_create(ctypes.byref(_shape(**change)), 4, 64, 1000, 0, ctypes.byref(h)) == status
    assert not h.value and L.xp_kv_last_error(None)


@pytest.mark.parametrize("batch,tokens,length,shared", [
    (0, 64, 100, 0), (4097, 64, 100, 0), (4, 0, 100, 0), (4, (1 << 20) + 1, 100, 0),
    (4, 64, 0, 0), (4, 64, (1 << 22) + 1, 0), (4, 64, 100, 2)])
def test_create_rejects_sizes(batch, tokens, length, shared):
    L = X.load_library()
    h = ctypes.c_void_p(0)
    s = _shape()
    assert L.xp_kv_create(ctypes.byref(s), batch, tokens, length, shared,
                          ctypes.byref(h)) == X.XP_EINVAL
    assert L.xp_kv_create(None, 4, 64, 100, 0, ctypes.byref(h)) == X.XP_EINVAL
    assert L.xp_kv_create(ctypes.byref(s), 4, 64, 100, 0, None) == X.XP_EINVAL


def test_null_handles_are_rejected():
    L = X.load_library()
    p = 0x1000                                     # never dereferenced
    assert L.xp_kv_map(None, 1, p, p, p, 4, p, p, p, p, p, p, 4, None) == X.XP_EINVAL
    assert L.xp_kv_write(None, 1, p, 1024, p, 1024, p, p, p, None, None, None) == X.XP_EINVAL
    attn = (p, 4096, None, p, p, 4, p, p, None, None, 1, 0, 0, 0.0, p, 4096, None, None)
    assert L.xp_kv_attn(None, 1, 1, 1, *attn) == X.XP_EINVAL
    assert L.xp_kv_attn_shared(None, 1, 1, 1, 1, p, p, *attn) == X.XP_EINVAL
    assert L.xp_kv_device_errors(None, None, None) == X.XP_EINVAL
    assert L.xp_layer_forward_paged(None, None, 1, 16, 1, 0, 0, p, p, p, None, None, p, 4, p, p, p,
                                    None) == X.XP_EINVAL
    L.xp_kv_destroy(None)
