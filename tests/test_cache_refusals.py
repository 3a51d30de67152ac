"""What the 4-bit cache refuses on the host, before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2607_20940_gb300 import msf

GOOD = dict(layers=1, kv_heads=2, head_dim=64, page_tokens=16, pages=8, sequences=3, sequence_pages=4)


def _cache(**kw):
    return msf.Cache(msf.make_cache_desc(**{**GOOD, **kw}))


@pytest.mark.parametrize("change,status", [
    (dict(layers=0), msf.MSF_ERR_INVALID_ARG), (dict(kv_heads=0), msf.MSF_ERR_INVALID_ARG),
    (dict(pages=0), msf.MSF_ERR_INVALID_ARG), (dict(pages=(1 << 24) + 1), msf.MSF_ERR_INVALID_ARG),
    (dict(sequences=0), msf.MSF_ERR_INVALID_ARG), (dict(sequences=65537), msf.MSF_ERR_INVALID_ARG),
    (dict(sequence_pages=0), msf.MSF_ERR_INVALID_ARG),
    (dict(sequence_pages=1 << 27), msf.MSF_ERR_INVALID_ARG),  # 2^31 tokens
    (dict(k_exponent=65), msf.MSF_ERR_INVALID_ARG), (dict(v_exponent=-65), msf.MSF_ERR_INVALID_ARG),
    (dict(head_dim=96), msf.MSF_ERR_UNSUPPORTED), (dict(page_tokens=24), msf.MSF_ERR_UNSUPPORTED),
    (dict(page_tokens=8), msf.MSF_ERR_UNSUPPORTED), (dict(page_tokens=256), msf.MSF_ERR_UNSUPPORTED),
])
def test_create(change, status):
    with pytest.raises(msf.MsfError) as e:
        _cache(**change)
    assert e.value.status == status


@pytest.mark.parametrize("D,P", [(64, 16), (128, 64)])
def test_sizes(D, P):
    info = _cache(head_dim=D, page_tokens=P, layers=3, kv_heads=5).info
    # keys and values: half a byte each, and a byte of scale for 16
    assert info.page_bytes == 5 * P * 2 * (D // 2 + D // 16)
    assert info.pool_bytes == 3 * 8 * info.page_bytes
    assert info.lengths_offset < info.table_offset < info.refs_offset < info.state_bytes


def _status(name, *args):
    return getattr(msf._lib, name)(*args)


def test_null_and_unbound():
    c = _cache()
    h, s3 = c.handle, (ctypes.c_int64 * 3)(0, 0, 0)
    a = msf.msf_cache_attention(heads=2, queries=1)
    assert _status("msf_cache_create", None, None) == msf.MSF_ERR_INVALID_ARG
    assert _status("msf_cache_query", None, None) == msf.MSF_ERR_INVALID_ARG
    assert _status("msf_cache_bind", h, None, 0, None, 0, None, 0) == msf.MSF_ERR_INVALID_ARG
    assert _status("msf_cache_bind", h, 256, 0, 256, 0, 256, 0) == msf.MSF_ERR_WORKSPACE
    assert _status("msf_cache_bind", h, 257, 1 << 40, 256, 1 << 40, 256, 1 << 40) == msf.MSF_ERR_INVALID_ARG
    for call in (("msf_cache_grow", None, None, 1, 1, None), ("msf_cache_write", 0, None, None, 1, 1, 16, 16, s3, None),
                 ("msf_cache_read", 0, None, None, 1, 1, 16, 16, s3, None), ("msf_cache_fork", 4, 4, None, 1, 0, None),
                 ("msf_cache_truncate", None, None, 1, None), ("msf_cache_compact", None),
                 ("msf_cache_attend", 0, None, 1, ctypes.byref(a), None),
                 ("msf_cache_attend_simt", 0, None, 1, ctypes.byref(a), None), ("msf_cache_device_status", None)):
        assert _status(call[0], None, *call[1:]) == msf.MSF_ERR_INVALID_ARG
        assert _status(call[0], h, *call[1:]) == msf.MSF_ERR_STATE
    msf.msf_cache_destroy(None)


def test_status_names():
    assert "pages" in msf.msf_status_string(msf.MSF_ERR_PAGES)
    assert "finite" in msf.msf_status_string(msf.MSF_ERR_NONFINITE)
