"""Pages of a paged cache against a plain model of the definitions (lists on the host)."""
import random

import pytest
import torch

from paper_2509_24257_b200 import binding as vb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Model:
    """The definitions, one sequence after the other."""

    def __init__(self, batch, width, n_pages, ps, layers):
        self.table, self.len, self.refs, self.ps, self.width = [[0] * width for _ in range(batch)], [0] * batch, [0] * n_pages, ps, width
        self.content = [[(-1 - p,) for p in range(n_pages)] for _ in range(layers)]  # what a page holds, by name
        self.short = False

    def have(self, n):
        return -(-n // self.ps)

    def reserve(self, new):
        growing = [b for b in range(len(new)) if self.len[b] < new[b] <= self.width * self.ps]
        free = [p for p, r in enumerate(self.refs) if r <= 0]
        at = 0
        holders = {}
        for b in growing:
            if self.len[b] % self.ps:
                holders.setdefault(self.table[b][self.have(self.len[b]) - 1], []).append(b)
        refs0 = list(self.refs)
        for b in growing:
            h = self.have(self.len[b])
            need = self.have(new[b]) - h
            copy = False
            if self.len[b] % self.ps:
                page = self.table[b][h - 1]
                keeps = len(holders[page]) == refs0[page] and holders[page][-1] == b
                copy = refs0[page] > 1 and not keeps
            if at + need + copy > len(free):
                self.short = True
                return
            if copy:
                page, to = self.table[b][h - 1], free[at]
                at += 1
                self.refs[page] -= 1
                self.refs[to] = 1
                self.table[b][h - 1] = to
                for c in self.content:
                    c[to] = c[page]
            for j in range(need):
                self.table[b][h + j] = free[at]
                self.refs[free[at]] = 1
                at += 1
            self.len[b] = new[b]

    def free(self, new):
        for b, n in enumerate(new):
            if 0 <= n < self.len[b]:
                for j in range(self.have(n), self.have(self.len[b])):
                    self.refs[self.table[b][j]] -= 1
                self.len[b] = n

    def fork(self, src, dst):
        lens, taken = list(self.len), set()
        for s, d in zip(src, dst):
            again = d in taken  # given before in this call, in a pair that was refused too
            taken.add(d)
            if not (0 <= s < len(lens) and 0 <= d < len(lens)) or lens[d] or again:
                continue
            for j in range(self.have(lens[s])):
                self.table[d][j] = self.table[s][j]
                self.refs[self.table[s][j]] += 1
            self.len[d] = lens[s]

    def compact(self):
        used = sum(r > 0 for r in self.refs)
        src = [p for p in range(used, len(self.refs)) if self.refs[p] > 0]
        dst = [p for p in range(used) if self.refs[p] <= 0]
        now = dict(zip(src, dst))
        for s, d in now.items():
            self.refs[d], self.refs[s] = self.refs[s], 0
            for c in self.content:
                c[d] = c[s]
        for b, n in enumerate(self.len):
            for j in range(self.have(n)):
                self.table[b][j] = now.get(self.table[b][j], self.table[b][j])
        return used


def _pages(batch, width, n_pages, ps, layers=2, heads=2, dim=64, dtype=torch.bfloat16, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = vb.KVPages.alloc(layers, batch, width, n_pages, ps, heads, dim, dtype, DEV)
    for c in h.caches:
        for t in (c.k, c.v):
            if t.element_size() == 2:
                t.copy_(torch.randn(t.shape, generator=g, device=DEV))
            else:
                t.view(torch.uint8).copy_(torch.randint(0, 120, t.shape, generator=g, device=DEV))
        for t in (c.k_scale, c.v_scale):
            if t is not None:
                t.copy_(torch.rand(t.shape, generator=g, device=DEV))
    return h, Model(batch, width, n_pages, ps, layers)


def _raw(c):
    return [t.view(torch.uint8).reshape(t.shape[0], -1).clone() for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]


def _same(h, m, start):
    """Tables, counts, lengths and the contents of the pages in use."""
    assert h.kv_len.tolist() == m.len
    assert [max(r, 0) for r in h.refs.tolist()] == m.refs
    table = h.page_table.tolist()
    for b, n in enumerate(m.len):
        assert table[b][:m.have(n)] == m.table[b][:m.have(n)], b
    used = [p for p, r in enumerate(m.refs) if r > 0]
    if used:
        for layer, c in enumerate(h.caches):
            was = [-1 - m.content[layer][p][0] for p in used]
            for now, then in zip(_raw(c), start[layer]):
                assert torch.equal(now[used], then[was])


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("batch,width,n_pages,ps", [(1, 1, 1, 16), (3, 5, 11, 16), (8, 40, 150, 32), (70, 9, 300, 16), (6, 3, 9, 256), (200, 30, 3000, 128)])
def test_random_histories(batch, width, n_pages, ps, dtype):
    r = random.Random(batch * 1000 + ps)
    h, m = _pages(batch, width, n_pages, ps, layers=r.choice([1, 3]), heads=r.choice([1, 3]), dtype=dtype)
    start = [_raw(c) for c in h.caches]
    cap = width * ps
    for step in range(24):
        kind = r.choice(["reserve", "reserve", "free", "fork", "compact"])
        if kind == "reserve":
            new = [min(cap, n + r.choice([0, 0, 1, 3, ps, cap])) if r.random() < 0.7 else r.randint(0, cap) for n in m.len]
            vb.kv_reserve(h, _i32(new))
            m.reserve(new)
        elif kind == "free":
            new = [r.choice([n, 0, max(0, n - 1), n // 2, n + 5]) for n in m.len]
            vb.kv_free(h, _i32(new))
            m.free(new)
        elif kind == "fork":
            empty = [b for b in range(batch) if m.len[b] == 0]
            r.shuffle(empty)
            dst = empty[:r.randint(0, len(empty))]
            src = [r.randrange(batch) for _ in dst]
            vb.kv_fork(h, _i32(src), _i32(dst))
            m.fork(src, dst)
        else:
            assert int(vb.kv_compact(h).item()) == m.compact()
        _same(h, m, start)
    assert int(h.status.item()) in ((0, vb.DEV_NO_PAGES) if m.short else (0,))
    vb.kv_free(h, _i32([0] * batch))
    assert sum(h.refs.tolist()) == 0 and h.kv_len.tolist() == [0] * batch


def test_the_last_holder_keeps_a_shared_page_and_the_others_get_copies():
    h, m = _pages(5, 4, 30, 16)
    start = [_raw(c) for c in h.caches]
    for op, model, args in ((vb.kv_reserve, m.reserve, ([20, 0, 0, 0, 0],)), (vb.kv_fork, m.fork, ([0, 0, 0], [1, 2, 4])),
                            (vb.kv_free, m.free, ([20, 18, 20, 0, 20],)), (vb.kv_reserve, m.reserve, ([21, 19, 0, 0, 40],)),
                            (vb.kv_reserve, m.reserve, ([22, 20, 21, 0, 41],))):
        op(h, *[_i32(a) for a in args])
        model(*args)
        _same(h, m, start)
    assert int(h.status.item()) == 0
    assert h.refs.tolist()[1] == 1  # the page that all shared: whoever came last has it to itself


def test_too_few_pages_serve_in_order_and_leave_the_rest():
    h, m = _pages(4, 8, 10, 16)
    start = [_raw(c) for c in h.caches]
    for new in ([40, 16, 0, 0], [100, 100, 17, 16], [41, 17, 16, 16]):
        vb.kv_reserve(h, _i32(new))
        m.reserve(new)
        _same(h, m, start)
    assert int(h.status.item()) == vb.DEV_NO_PAGES
    with pytest.raises(RuntimeError):
        h.check()


def test_a_keeper_is_not_served_when_a_copy_before_it_was_not():
    h, m = _pages(2, 4, 2, 16)
    start = [_raw(c) for c in h.caches]
    for op, model, args in ((vb.kv_reserve, m.reserve, ([20, 0],)), (vb.kv_fork, m.fork, ([0], [1])), (vb.kv_reserve, m.reserve, ([21, 21],))):
        op(h, *[_i32(a) for a in args])
        model(*args)
        _same(h, m, start)
    assert h.kv_len.tolist() == [20, 20] and h.refs.tolist() == [2, 2] and int(h.status.item()) == vb.DEV_NO_PAGES


def test_bad_lengths_pages_and_pairs_are_reported_and_bounded():
    def fresh():
        h, m = _pages(4, 4, 12, 16)
        vb.kv_reserve(h, _i32([20, 5, 0, 0]))
        m.reserve([20, 5, 0, 0])
        return h, m, [_raw(c) for c in h.caches]

    h, m, start = fresh()
    vb.kv_reserve(h, _i32([65, 6, -4, 2 ** 31 - 1]))  # beyond the table's row
    m.reserve([20, 6, 0, 0])
    _same(h, m, start)
    assert int(h.status.item()) == vb.DEV_ROWS_RANGE
    h, m, start = fresh()
    vb.kv_free(h, _i32([-1, 3, 0, 7]))
    m.free([20, 3, 0, 0])
    _same(h, m, start)
    assert int(h.status.item()) == vb.DEV_ROWS_RANGE
    h, m, start = fresh()
    pairs = ([0, 0, 9, 1, -1, 0, 1], [2, 2, 3, 0, 3, 7, 3])  # given twice, out of range, not empty
    h4 = h
    for i in range(0, 7, 4):
        vb.kv_fork(h4, _i32(pairs[0][i:i + 4]), _i32(pairs[1][i:i + 4]))
        m.fork(pairs[0][i:i + 4], pairs[1][i:i + 4])
        _same(h, m, start)
    assert int(h.status.item()) == vb.DEV_ROWS_RANGE
    h, m, start = fresh()
    h.page_table[0, 1] = 12  # the page that would be copied or dropped
    vb.kv_reserve(h, _i32([21, 6, 0, 0]))
    vb.kv_free(h, _i32([1, 1, 0, 0]))
    assert int(h.status.item()) == vb.DEV_PAGE_RANGE and h.kv_len.tolist() == [1, 1, 0, 0] and sum(h.refs.tolist()) == 3
    h, m, start = fresh()
    h.kv_len[1] = 1000  # bounded to the row of the table
    vb.kv_free(h, _i32([20, 999, 0, 0]))
    assert int(h.status.item()) == vb.DEV_ROWS_RANGE


def test_forking_an_empty_or_the_same_sequence():
    h, m = _pages(3, 2, 4, 16)
    vb.kv_fork(h, _i32([0, 1]), _i32([1, 0]))
    vb.kv_fork(h, _i32([2]), _i32([2]))
    assert h.kv_len.tolist() == [0, 0, 0] and h.refs.tolist() == [0] * 4 and int(h.status.item()) == 0
    vb.kv_fork(h, _i32([]), _i32([]))


def test_many_pages_and_long_rows():
    """More pages than one step of the scan looks at, more sequences than the CTA has threads."""
    n_pages, batch, width, ps = 70000, 1500, 60, 16
    h, m = _pages(batch, width, n_pages, ps, layers=1, heads=1)
    start = [_raw(c) for c in h.caches]
    r = random.Random(4)
    new = [r.randint(0, width * ps) for _ in range(batch)]
    vb.kv_reserve(h, _i32(new))
    m.reserve(new)
    new = [n if b % 3 else 0 for b, n in enumerate(m.len)]
    vb.kv_free(h, _i32(new))
    m.free(new)
    src = [b + 1 for b in range(0, 1200, 3)]
    dst = [b for b in range(0, 1200, 3)]
    vb.kv_fork(h, _i32(src), _i32(dst))
    m.fork(src, dst)
    new = [min(width * ps, n + 3) if n else 0 for n in m.len]
    vb.kv_reserve(h, _i32(new))
    m.reserve(new)
    _same(h, m, start)
    vb.kv_free(h, _i32([n if b % 2 else 0 for b, n in enumerate(m.len)]))
    m.free([n if b % 2 else 0 for b, n in enumerate(m.len)])
    assert int(vb.kv_compact(h).item()) == m.compact()
    _same(h, m, start)
    assert int(h.status.item()) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("ps,heads,dim", [(16, 1, 64), (64, 8, 128), (256, 3, 64)])
def test_copy_between_pools(dtype, ps, heads, dim):
    a, _ = _pages(1, 1, 9, ps, 3, heads, dim, dtype, 1)
    b, _ = _pages(1, 1, 14, ps, 3, heads, dim, dtype, 2)
    before = [_raw(c) for c in b.caches]
    src, dst = [3, 0, -1, 8, 3, 5], [13, 2, 4, 0, 6, -1]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    vb.kv_copy(a.caches, b.caches, _i32(src), _i32(dst), status=status)
    for ca, cb, was in zip(a.caches, b.caches, before):
        want = [w.clone() for w in was]
        for s, d in zip(src, dst):
            if s >= 0 and d >= 0:
                for w, x in zip(want, _raw(ca)):
                    w[d] = x[s]
        assert all(torch.equal(x, y) for x, y in zip(_raw(cb), want))
    assert int(status.item()) == 0
    vb.kv_copy(a.caches, b.caches, _i32([9, 1, -2]), _i32([1, 14, 1]), status=status)
    assert int(status.item()) == vb.DEV_PAGE_RANGE
    assert all(torch.equal(x, y) for c, y_ in zip(b.caches[:1], [want]) for x, y in zip(_raw(b.caches[-1]), want))
    vb.kv_copy(a.caches, a.caches, _i32([0]), _i32([1]))
    assert all(torch.equal(x[0], x[1]) for c in a.caches for x in _raw(c))


@pytest.mark.parametrize("layers,dtype", [(1, torch.bfloat16), (3, torch.int8), (7, torch.float8_e4m3fn)])
def test_more_pages_to_copy_than_run_at_once(layers, dtype):
    a, _ = _pages(1, 1, 3000, 16, layers, 1, 64, dtype, 1)
    b, _ = _pages(1, 1, 3500, 16, layers, 1, 64, dtype, 2)
    g = torch.Generator().manual_seed(5)
    src, dst = torch.randint(-1, 3000, (3400,), generator=g, dtype=torch.int32), torch.randperm(3500, generator=g)[:3400].to(torch.int32)
    want = [[w.clone() for w in _raw(c)] for c in b.caches]
    ok = src >= 0
    for ca, ws in zip(a.caches, want):
        for w, x in zip(ws, _raw(ca)):
            w[dst[ok].long().to(DEV)] = x[src[ok].long().to(DEV)]
    vb.kv_copy(a.caches, b.caches, src.to(DEV), dst.to(DEV))
    assert all(torch.equal(x, y) for c, ws in zip(b.caches, want) for x, y in zip(_raw(c), ws))


def test_pools_beyond_four_gigabytes():
    ps, heads, dim, n = 256, 8, 128, 9000  # 4.7 GB per pool
    k = torch.zeros(n, heads, ps, dim, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros(n, heads, ps, dim, dtype=torch.bfloat16, device=DEV)
    cache = vb.KVCache(k, v)
    k[8999].fill_(3.0)
    v[8999].fill_(4.0)
    refs = torch.zeros(n, dtype=torch.int32, device=DEV)
    refs[8999] = 2
    h = vb.KVPages([cache], _i32([[8999, 0], [8999, 0]]), _i32([100, 100]), refs)
    vb.kv_reserve(h, _i32([101, 100]))
    assert h.page_table.tolist() == [[0, 0], [8999, 0]] and float(k[0].mean()) == 3.0 and float(v[0].mean()) == 4.0
    vb.kv_copy([cache], [cache], _i32([8999]), _i32([8998]))
    assert float(k[8998].mean()) == 3.0
    assert int(vb.kv_compact(h).item()) == 2
    assert h.page_table.tolist() == [[0, 0], [1, 0]] and float(v[1].mean()) == 4.0 and float(k[8998].mean()) == 3.0


def test_a_captured_step_follows_the_tables_contents():
    h, m = _pages(6, 12, 80, 16, layers=2)
    start = [_raw(c) for c in h.caches]
    first = [30, 5, 64, 1, 0, 0]
    vb.kv_reserve(h, _i32(first))
    m.reserve(first)
    vb.kv_fork(h, _i32([0]), _i32([4]))
    m.fork([0], [4])
    grow, keep, used = _i32([0] * 6), _i32([0] * 6), None
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.kv_reserve(h, grow)
        vb.kv_free(h, keep)
        used = vb.kv_compact(h)
    for step in range(6):
        new = [n + 5 if n else 0 for n in m.len]
        final = [n + 1 + step % 4 if n else 0 for n in m.len]
        grow.copy_(_i32(new))
        keep.copy_(_i32(final))
        graph.replay()
        m.reserve(new)
        m.free(final)
        assert int(used.item()) == m.compact()
        _same(h, m, start)
    h.check()


def test_on_another_stream():
    h, m = _pages(6, 12, 80, 16)
    start = [_raw(c) for c in h.caches]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    new, more = _i32([50, 20, 3, 0, 0, 0]), _i32([51, 21, 4, 51, 0, 0])
    src, dst = _i32([0]), _i32([3])
    side.wait_stream(torch.cuda.current_stream())
    vb.kv_reserve(h, new, stream=side)
    vb.kv_fork(h, src, dst, stream=side)
    vb.kv_reserve(h, more, stream=side)
    used = vb.kv_compact(h, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    m.reserve(new.tolist())
    m.fork([0], [3])
    m.reserve(more.tolist())
    assert int(used.item()) == m.compact()
    _same(h, m, start)


def test_refusals():
    h, _ = _pages(3, 4, 10, 16)
    for bad in (_i32([1, 2]), torch.ones(3, device=DEV), torch.ones(3, dtype=torch.int32)):
        with pytest.raises(ValueError):
            vb.kv_reserve(h, bad)
        with pytest.raises(ValueError):
            vb.kv_free(h, bad)
    with pytest.raises(ValueError):
        vb.kv_fork(h, _i32([0]), _i32([1, 2]))
    with pytest.raises(vb.VerillmError):
        vb.kv_fork(h, _i32([0] * 4), _i32([1] * 4))  # more pairs than sequences
    with pytest.raises(ValueError):
        vb.KVPages([], h.page_table, h.kv_len, h.refs)
    with pytest.raises(ValueError):
        vb.KVPages(h.caches, h.page_table, h.kv_len, h.refs[:5])
    other, _ = _pages(3, 4, 10, 32)
    with pytest.raises(vb.VerillmError):
        vb.kv_copy(h.caches, other.caches, _i32([0]), _i32([1]))
    with pytest.raises(ValueError):
        vb.kv_copy(h.caches, other.caches[:1], _i32([0]), _i32([1]))
    mixed = vb.KVPages([h.caches[0], other.caches[0]], h.page_table, h.kv_len, h.refs)
    with pytest.raises(vb.VerillmError):
        vb.kv_reserve(mixed, _i32([1, 1, 1]))
