"""Which calls of the paged attention are split over CTAs and joined, and that both ways give the definition (needs a B200)."""
import pytest
import torch

from paper_2509_24257_b200 import binding as vb
from tests.paged_cases import Case, assert_within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, E4M3, INT8 = torch.bfloat16, torch.float8_e4m3fn, torch.int8
DTYPES = [BF16, E4M3, INT8]


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_short_context_alone_is_split_over_the_gpu(dtype):
    """One sequence of 500 positions has a block per kv head: in one piece it would leave nearly all CTAs idle.  A batch
    whose blocks fill the GPU is not split.  (A split call leaves partial results in its workspace.)"""
    for batch, positions, split in ((1, 500, True), (4, 500, True), (60, 500, False), (1, 250, False), (60, 700, True)):
        c = Case(dtype, 16, 4, 64, 16, [1] * batch, [positions] * batch, seed=50, pad=0, width_extra=0)
        cache, rows = c.device()
        ws = torch.full((1 << 24,), 0xFF, dtype=torch.uint8, device=DEV)
        got = vb.op_attention_paged(c.dq, cache, rows, workspace=ws)
        rows.check()
        assert bool((ws != 0xFF).any()) == split, (batch, positions)
        ref, tol, _, _ = c.attention()
        assert_within(got.reshape(c.n, 16, 64), ref, tol)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 3])
def test_workspaces_of_larger_batches_serve_smaller_ones(dtype, rows):
    """Fewer sequences may be split where more are not; what the workspace holds before the call does not matter."""
    for kv in (250, 500, 520, 1000):
        needs = []
        for batch in (1, 4, 9, 10, 19, 64, 80, 200):
            c = Case(dtype, 8, 8, 64, 16, [rows] * batch, [kv] * batch, seed=51, pad=0, width_extra=0)
            cache, r = c.device()
            needs.append(vb.attention_paged_workspace(cache, r, c.n, 8))
            if batch in (1, 9, 10, 19, 64):
                got = vb.op_attention_paged(c.dq, cache, r)
                ws = torch.full((max(needs[-1], 1),), 0xFF, dtype=torch.uint8, device=DEV)
                assert torch.equal(got, vb.op_attention_paged(c.dq, cache, r, workspace=ws))
                r.check()
                if kv == 500 and batch != 64:
                    ref, tol, _, _ = c.attention()
                    assert_within(got.reshape(c.n, 8, 64), ref, tol)
        assert all(a <= b for a, b in zip(needs, needs[1:])), (kv, needs)


def test_any_bound_on_the_rows_is_taken_as_it_is():
    """A bound beyond 32 bits is a bound: cut off, it would be a small one and the sequences skipped."""
    c = Case(E4M3, 4, 2, 64, 16, [7, 2], [40, 30], seed=52, pad=0)
    cache, rows = c.device()
    want = vb.op_attention_paged(c.dq, cache, rows)
    for most in (1 << 31, (1 << 32) + 1, 1 << 40):
        wide = vb.PagedRows(rows.page_table, rows.cu_rows, rows.kv_len, most, rows.status)
        assert torch.equal(vb.op_attention_paged(c.dq, cache, wide), want)
        wide.check()
