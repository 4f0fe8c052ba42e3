"""Refusals of the 4-bit, draft and page entry points: all made on the host, before a device is touched."""
import ctypes as C

import pytest

from paper_2509_24257_b200 import binding as vb
from paper_2509_24257_b200 import build

PTR = 1 << 20  # stands for a device pointer; nothing is launched


@pytest.fixture(scope="module")
def library():
    build.build_library()
    return vb.lib()


def _w4(**kw):
    f = dict(codes=PTR, scales=PTR, n=64, k=256, group=128)
    f.update(kw)
    return vb.W4C(**f)


@pytest.mark.parametrize("kw,code", [
    (dict(codes=None), vb.E_INVAL), (dict(scales=None), vb.E_INVAL), (dict(n=0), vb.E_INVAL), (dict(k=-128), vb.E_INVAL), (dict(group=16), vb.E_SHAPE),
    (dict(group=256), vb.E_SHAPE), (dict(k=192), vb.E_SHAPE), (dict(n=60), vb.E_SHAPE), (dict(codes=PTR + 8), vb.E_SHAPE), (dict(scales=PTR + 2), vb.E_SHAPE)])
def test_bad_weights_are_refused(library, kw, code):
    w = C.byref(_w4(**kw))
    assert library.verillm_w4_quantise(PTR, 256, w, None) == code
    assert library.verillm_w4_dequantise(w, PTR, 256, vb.F32, None) == code
    assert library.verillm_op_w4_matvec(w, PTR, 256, 1, None, 0, PTR + 4096, 64, vb.F32, None, None) == code


def test_bad_matrices_are_refused(library):
    w = C.byref(_w4())
    for fn in (lambda p, s: library.verillm_w4_quantise(p, s, w, None), lambda p, s: library.verillm_w4_dequantise(w, p, s, vb.BF16, None),
               lambda p, s: library.verillm_op_w4_matvec(w, p, s, 2, None, 0, PTR + (1 << 16), 64, vb.BF16, None, None)):
        assert fn(None, 256) == vb.E_INVAL
        assert fn(PTR + 8, 256) == vb.E_SHAPE and fn(PTR, 248) == vb.E_SHAPE and fn(PTR, 260) == vb.E_SHAPE
    y = PTR + (1 << 16)
    call = library.verillm_op_w4_matvec
    assert library.verillm_w4_dequantise(w, PTR, 256, 2, None) == vb.E_INVAL
    assert call(w, PTR, 256, -1, None, 0, y, 64, vb.F32, None, None) == vb.E_INVAL
    assert call(w, PTR, 256, 1, None, 0, y, 64, 5, None, None) == vb.E_INVAL
    assert call(w, PTR, 256, 1, None, 0, None, 64, vb.F32, None, None) == vb.E_INVAL
    assert call(w, PTR, 256, 1, None, 0, PTR, 64, vb.F32, None, None) == vb.E_INVAL  # y over x
    assert call(w, PTR, 256, 1, None, 0, y + 2, 64, vb.F32, None, None) == vb.E_SHAPE
    assert call(w, PTR, 256, 1, None, 0, y, 63, vb.F32, None, None) == vb.E_SHAPE
    assert call(w, PTR, 256, 1, PTR * 4, 63, y, 64, vb.F32, None, None) == vb.E_SHAPE
    assert call(w, PTR, 256, 1, y, 64, y, 64, vb.BF16, None, None) == vb.E_INVAL  # the residual as a bf16 output
    assert call(w, PTR, 256, 1, y, 72, y, 64, vb.F32, None, None) == vb.E_INVAL
    assert call(w, PTR, 256, 65537, None, 0, y, 64, vb.F32, None, None) == vb.E_SHAPE
    assert call(w, None, 0, 0, None, 0, None, 0, vb.F32, None, None) == 0  # no rows: nothing to do


def _drafts(**kw):
    f = dict(target=PTR, draft=PTR, target_stride=100, draft_stride=100, dtype=vb.F32, vocab=100, batch=2, n_rows=5, max_rows=4, cu_rows=PTR, tokens=PTR,
             kv_len=PTR, temperature=PTR, accept_u=PTR, sample_u=PTR)
    f.update(kw)
    return vb.DraftsC(**f)


def _report(**kw):
    f = dict(tokens=PTR, n_emitted=PTR, logp=PTR, new_len=PTR)
    f.update(kw)
    return vb.DraftReportC(**f)


@pytest.mark.parametrize("kw,code", [
    (dict(target=None), vb.E_INVAL), (dict(tokens=None), vb.E_INVAL), (dict(cu_rows=None), vb.E_INVAL), (dict(accept_u=None), vb.E_INVAL),
    (dict(sample_u=None), vb.E_INVAL), (dict(kv_len=None), vb.E_INVAL), (dict(batch=0), vb.E_INVAL), (dict(n_rows=-1), vb.E_INVAL),
    (dict(max_rows=0), vb.E_INVAL), (dict(vocab=0), vb.E_INVAL), (dict(dtype=2), vb.E_INVAL), (dict(max_rows=257), vb.E_SHAPE),
    (dict(vocab=(1 << 24) + 1), vb.E_SHAPE), (dict(target_stride=99), vb.E_SHAPE), (dict(draft_stride=99), vb.E_SHAPE), (dict(target=PTR + 2), vb.E_SHAPE),
    (dict(draft=PTR + 1, dtype=vb.BF16), vb.E_SHAPE)])
def test_bad_drafts_are_refused(library, kw, code):
    assert library.verillm_verify_drafts(C.byref(_drafts(**kw)), C.byref(_report()), PTR, 1 << 30, None, None) == code


def test_bad_reports_and_workspaces_are_refused(library):
    d, call = C.byref(_drafts()), library.verillm_verify_drafts
    assert call(None, C.byref(_report()), PTR, 1 << 30, None, None) == vb.E_INVAL
    assert call(d, None, PTR, 1 << 30, None, None) == vb.E_INVAL
    assert call(d, C.byref(_report(tokens=None)), PTR, 1 << 30, None, None) == vb.E_INVAL
    assert call(d, C.byref(_report(n_emitted=None)), PTR, 1 << 30, None, None) == vb.E_INVAL
    assert call(d, C.byref(_report()), None, 1 << 30, None, None) == vb.E_INVAL
    assert call(d, C.byref(_report()), PTR + 8, 1 << 30, None, None) == vb.E_SHAPE
    assert call(d, C.byref(_report()), PTR, library.verillm_verify_drafts_workspace(5) - 1, None, None) == vb.E_SHAPE
    assert library.verillm_verify_drafts_workspace(-1) == vb.E_INVAL


def test_reports_over_their_inputs_are_refused(library):
    call = library.verillm_verify_drafts
    apart = dict(tokens=PTR + (1 << 20), logp=PTR + (2 << 20))
    for kw in (dict(tokens=PTR), dict(logp=PTR)):
        assert call(C.byref(_drafts()), C.byref(_report(**dict(apart, **kw))), PTR, 1 << 30, None, None) == vb.E_INVAL


def test_no_layers_to_copy():
    with pytest.raises(ValueError):
        vb.kv_copy([], [], None, None)


def _layers(n=2, **kw):
    f = dict(k=PTR, v=PTR, k_scale=PTR, v_scale=PTR, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, dtype=vb.KV_E4M3)
    a = [dict(f) for _ in range(n)]
    a[-1].update(kw)
    return (vb.KVCacheC * n)(*[vb.KVCacheC(**x) for x in a])


def _pages(layers=None, **kw):
    layers = layers if layers is not None else _layers()
    f = dict(layers=layers, n_layers=len(layers), page_table=PTR, kv_len=PTR, refs=PTR, batch=2, table_width=4)
    f.update(kw)
    return vb.KVPagesC(**f)


def _codes(library, pages, ws=PTR, ws_bytes=1 << 30):
    p = C.byref(pages)
    return [library.verillm_kv_reserve(p, PTR, ws, ws_bytes, None, None), library.verillm_kv_fork(p, PTR, PTR, 1, ws, ws_bytes, None, None),
            library.verillm_kv_compact(p, PTR, ws, ws_bytes, None, None)]


@pytest.mark.parametrize("kw,code", [
    (dict(page_table=None), vb.E_INVAL), (dict(kv_len=None), vb.E_INVAL), (dict(refs=None), vb.E_INVAL), (dict(batch=0), vb.E_INVAL),
    (dict(table_width=0), vb.E_INVAL), (dict(n_layers=0), vb.E_INVAL), (dict(n_layers=129), vb.E_SHAPE), (dict(table_width=(1 << 22) + 1), vb.E_SHAPE)])
def test_bad_pages_are_refused(library, kw, code):
    pages = _pages(**kw)
    assert _codes(library, pages) == [code] * 3
    assert library.verillm_kv_free(C.byref(pages), PTR, None, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), vb.E_INVAL), (dict(v_scale=None), vb.E_INVAL), (dict(dtype=7), vb.E_INVAL), (dict(n_pages=11), vb.E_SHAPE), (dict(page_size=32), vb.E_SHAPE),
    (dict(n_kv_heads=4), vb.E_SHAPE), (dict(head_dim=128), vb.E_SHAPE), (dict(dtype=vb.KV_INT8), vb.E_SHAPE), (dict(k=PTR + 16), vb.E_SHAPE)])
def test_layers_of_another_geometry_are_refused(library, kw, code):
    layers = _layers(**kw)
    assert _codes(library, _pages(layers)) == [code] * 3
    good = _layers()
    assert library.verillm_kv_copy(layers, good, 2, PTR, PTR, 1, None, None) == code
    assert library.verillm_kv_copy(good, layers, 2, PTR, PTR, 1, None, None) == code


def test_workspaces_lists_and_counts_are_checked(library):
    need = library.verillm_kv_pages_workspace(2, 10)
    assert need > 0 and library.verillm_kv_pages_workspace(0, 10) == vb.E_INVAL and library.verillm_kv_pages_workspace(2, 0) == vb.E_INVAL
    assert _codes(library, _pages(), None) == [vb.E_INVAL] * 3
    assert _codes(library, _pages(), PTR + 4) == [vb.E_SHAPE] * 3
    assert _codes(library, _pages(), PTR, need - 1) == [vb.E_SHAPE] * 3
    p = C.byref(_pages())
    assert library.verillm_kv_reserve(p, None, PTR, need, None, None) == vb.E_INVAL
    assert library.verillm_kv_free(p, None, None, None) == vb.E_INVAL
    assert library.verillm_kv_compact(p, None, PTR, need, None, None) == vb.E_INVAL
    assert library.verillm_kv_fork(p, None, PTR, 1, PTR, need, None, None) == vb.E_INVAL
    assert library.verillm_kv_fork(p, PTR, PTR, 3, PTR, need, None, None) == vb.E_SHAPE
    assert library.verillm_kv_fork(p, PTR, PTR, -1, PTR, need, None, None) == vb.E_INVAL
    assert library.verillm_kv_fork(p, None, None, 0, None, 0, None, None) == 0
    a = _layers()
    assert library.verillm_kv_copy(a, a, 2, None, None, 0, None, None) == 0
    assert library.verillm_kv_copy(a, a, 2, None, PTR, 1, None, None) == vb.E_INVAL
    assert library.verillm_kv_copy(a, _layers(page_size=32, n=1), 1, PTR, PTR, 1, None, None) == vb.E_SHAPE
    assert library.verillm_kv_copy(None, a, 2, PTR, PTR, 1, None, None) == vb.E_INVAL
