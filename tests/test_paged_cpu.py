"""Refusals of the paged-cache entry points: all made on the host, before a device is touched."""
import ctypes as C

import pytest

from paper_2509_24257_b200 import binding as vb
from paper_2509_24257_b200 import build

PTR = 1 << 20  # stands for a device pointer; nothing is launched


@pytest.fixture(scope="module")
def library():
    build.build_library()
    return vb.lib()


def _cache(**kw):
    f = dict(k=PTR, v=PTR, k_scale=PTR, v_scale=PTR, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, dtype=vb.KV_E4M3)
    f.update(kw)
    return vb.KVCacheC(**f)


def _rows(**kw):
    f = dict(page_table=PTR, cu_rows=PTR, kv_len=PTR, table_width=4, batch=2, n_rows=3, max_rows=2)
    f.update(kw)
    return vb.KVRowsC(**f)


def _codes(library, cache, rows):
    """What the four entry points answer."""
    c, r = C.byref(cache), C.byref(rows)
    return [
        library.verillm_kv_write(c, r, PTR, PTR, 128, None, None),
        library.verillm_kv_read(c, r, PTR, PTR, 128, vb.F32, None, None),
        library.verillm_op_attention_paged(c, r, PTR, 256, 4, PTR, 256, None, PTR, 1 << 40, None, None),
        library.verillm_op_attention_paged_workspace(c, r, 4),
    ]


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), vb.E_INVAL), (dict(v=None), vb.E_INVAL), (dict(k_scale=None), vb.E_INVAL), (dict(v_scale=None), vb.E_INVAL),
    (dict(dtype=3), vb.E_INVAL), (dict(dtype=-1), vb.E_INVAL), (dict(n_pages=0), vb.E_INVAL), (dict(n_kv_heads=0), vb.E_INVAL),
    (dict(page_size=8), vb.E_SHAPE), (dict(page_size=48), vb.E_SHAPE), (dict(page_size=512), vb.E_SHAPE), (dict(page_size=0), vb.E_SHAPE),
    (dict(head_dim=96), vb.E_SHAPE), (dict(head_dim=256), vb.E_SHAPE), (dict(k=PTR + 8), vb.E_SHAPE), (dict(v=PTR + 1), vb.E_SHAPE), (dict(k=PTR + 16), vb.E_SHAPE), (dict(v=PTR + 16), vb.E_SHAPE), (dict(k_scale=PTR + 4), vb.E_SHAPE), (dict(v_scale=PTR + 8), vb.E_SHAPE),
    (dict(n_pages=1 << 27, page_size=16, n_kv_heads=2), vb.E_SHAPE),  # rows beyond 32 bits
])
def test_bad_caches_are_refused(library, kw, code):
    assert _codes(library, _cache(**kw), _rows()) == [code] * 4


@pytest.mark.parametrize("kw", [dict(page_table=None), dict(cu_rows=None), dict(kv_len=None), dict(table_width=0), dict(batch=0),
                                dict(n_rows=-1), dict(max_rows=0)])
def test_bad_rows_are_refused(library, kw):
    assert _codes(library, _cache(), _rows(**kw)) == [vb.E_INVAL] * 4


def test_bad_matrices_are_refused(library):
    c, r = C.byref(_cache()), C.byref(_rows())
    for fn in (lambda p, q, s: library.verillm_kv_write(c, r, p, q, s, None, None),
               lambda p, q, s: library.verillm_kv_read(c, r, p, q, s, vb.BF16, None, None),
               lambda p, q, s: library.verillm_op_attention_paged(c, r, p, s, 2, q, s, None, PTR, 1 << 40, None, None)):
        assert fn(None, PTR, 128) == vb.E_INVAL and fn(PTR, None, 128) == vb.E_INVAL
        assert fn(PTR + 8, PTR, 128) == vb.E_SHAPE and fn(PTR, PTR + 2, 128) == vb.E_SHAPE
        assert fn(PTR, PTR, 120) == vb.E_SHAPE  # rows would overlap
        assert fn(PTR, PTR, 132) == vb.E_SHAPE  # rows not 16-byte aligned
    assert library.verillm_kv_read(c, r, PTR, PTR, 128, 2, None, None) == vb.E_INVAL
    for heads, code in ((0, vb.E_INVAL), (-2, vb.E_INVAL), (3, vb.E_SHAPE), (2 * 129, vb.E_SHAPE)):
        assert library.verillm_op_attention_paged(c, r, PTR, 1 << 20, heads, PTR, 1 << 20, None, PTR, 1 << 40, None, None) == code
        assert library.verillm_op_attention_paged_workspace(c, r, heads) == code


def test_no_rows_is_a_no_op_without_a_device(library):
    c, r = C.byref(_cache()), C.byref(_rows(n_rows=0))
    assert library.verillm_kv_write(c, r, None, None, 0, None, None) == 0
    assert library.verillm_kv_read(c, r, None, None, 0, vb.BF16, None, None) == 0
    assert library.verillm_op_attention_paged(c, r, None, 0, 4, None, 0, None, None, 0, None, None) == 0


def test_null_descriptions_are_refused(library):
    assert library.verillm_kv_write(None, None, PTR, PTR, 128, None, None) == vb.E_INVAL
    assert library.verillm_kv_read(None, None, PTR, PTR, 128, 0, None, None) == vb.E_INVAL
    assert library.verillm_op_attention_paged(None, None, PTR, 256, 4, PTR, 256, None, PTR, 0, None, None) == vb.E_INVAL
    assert library.verillm_op_attention_paged_workspace(None, None, 4) == vb.E_INVAL


def test_contexts_beyond_the_bound_and_output_over_the_queries_are_refused(library):
    cache = _cache(page_size=256, n_pages=1 << 18)
    assert _codes(library, cache, _rows(table_width=(1 << 18) + 1)) == [vb.E_SHAPE] * 4
    c, r = C.byref(cache), C.byref(_rows())
    assert library.verillm_op_attention_paged(c, r, PTR, 256, 4, PTR, 256, None, PTR, 1 << 40, None, None) == vb.E_INVAL
