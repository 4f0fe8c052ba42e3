"""Page calls through holders that live no longer than the call, on other streams and captured."""
import gc

import pytest
import torch

from paper_2509_24257_b200 import binding as vb
from tests.test_gpu_pages import _i32, _pages, _raw, _same

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _again(h):
    return vb.KVPages(h.caches, h.page_table, h.kv_len, h.refs, h.status)


def _litter(h):
    """Tensors of the current stream where a workspace that was let go may have been."""
    return [torch.full((h._ws_bytes // 4,), v, dtype=torch.int32, device=DEV) for v in (3, 1 << 30, 5, -1) for _ in range(4)]


def test_a_holder_made_for_one_call_on_a_busy_stream():
    h, m = _pages(6, 12, 80, 16)
    start = [_raw(c) for c in h.caches]
    side = torch.cuda.Stream()
    new, more, last = _i32([50, 20, 3, 0, 0, 0]), _i32([51, 21, 4, 51, 52, 0]), _i32([9, 21, 0, 51, 52, 0])
    src, dst = _i32([0, 0]), _i32([3, 4])
    side.wait_stream(torch.cuda.current_stream())
    keep = []
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    vb.kv_reserve(_again(h), new, stream=side)
    keep.append(_litter(h))
    vb.kv_fork(_again(h), src, dst, stream=side)
    keep.append(_litter(h))
    vb.kv_reserve(_again(h), more, stream=side)
    keep.append(_litter(h))
    vb.kv_free(_again(h), last, stream=side)
    used = vb.kv_compact(_again(h), stream=side)
    keep.append(_litter(h))
    with torch.cuda.stream(side):  # the same by the current stream
        more2 = _i32([60, 21, 4, 51, 64, 3])
        vb.kv_reserve(_again(h), more2)
    keep.append(_litter(h))
    torch.cuda.synchronize()
    m.reserve(new.tolist())
    m.fork([0, 0], [3, 4])
    m.reserve(more.tolist())
    m.free(last.tolist())
    assert int(used.item()) == m.compact()
    m.reserve(more2.tolist())
    _same(h, m, start)
    h.check()


@pytest.mark.parametrize("made_on_the_same_stream", [False, True])
def test_a_captured_step_outlives_its_holder(made_on_the_same_stream):
    h, m = _pages(6, 12, 80, 16)
    start = [_raw(c) for c in h.caches]
    vb.kv_reserve(h, _i32([30, 5, 64, 1, 0, 0]))
    m.reserve([30, 5, 64, 1, 0, 0])
    vb.kv_fork(h, _i32([0]), _i32([4]))
    m.fork([0], [4])
    grow, cut = _i32([0] * 6), _i32([0] * 6)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side if made_on_the_same_stream else torch.cuda.current_stream()):
        holder = _again(h)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        vb.kv_reserve(holder, grow)
        vb.kv_free(holder, cut)
        used = vb.kv_compact(holder)
    del holder
    gc.collect()
    litter = _litter(h)
    with torch.cuda.stream(side):
        litter += _litter(h)
    torch.cuda.synchronize()
    for step in range(4):
        new = [n + 5 if n else 0 for n in m.len]
        final = [n + 1 + step % 4 if n else 0 for n in m.len]
        grow.copy_(_i32(new))
        cut.copy_(_i32(final))
        graph.replay()
        m.reserve(new)
        m.free(final)
        assert int(used.item()) == m.compact()
        _same(h, m, start)
    torch.cuda.synchronize()
    values = (3, 1 << 30, 5, -1)
    assert all(bool((t == values[i // 4 % 4]).all()) for i, t in enumerate(litter))  # nor does it write where it may not
    h.check()
