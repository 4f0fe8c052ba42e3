"""The counts of table entries per page, as they are: none below 0, none left over."""
import random

import pytest
import torch

from paper_2509_24257_b200 import binding as vb
from tests.test_gpu_pages import _i32, _pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("batch,width,n_pages,ps", [(3, 5, 11, 16), (8, 40, 150, 32), (70, 9, 300, 16), (1100, 6, 2500, 16)])
def test_counts_are_those_of_the_table(batch, width, n_pages, ps, seed):
    r = random.Random(batch + seed)
    h, m = _pages(batch, width, n_pages, ps, layers=1, heads=1)
    cap = width * ps
    for step in range(20):
        kind = r.choice(["reserve", "reserve", "free", "fork", "fork", "compact"])
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
        refs, table, lens = h.refs.tolist(), h.page_table.tolist(), h.kv_len.tolist()
        assert refs == m.refs and lens == m.len
        held = [0] * n_pages
        for row, n in zip(table, lens):
            for page in row[:-(-n // ps)]:
                held[page] += 1
        assert refs == held
    vb.kv_free(h, _i32([0] * batch))
    assert h.refs.tolist() == [0] * n_pages and h.kv_len.tolist() == [0] * batch
