"""Kernels whose CTAs work in clusters, where the threads of a warp take different ways to the last barrier."""
import pytest
import torch

from paper_2509_24257_b200 import binding as vb
from tests.test_gpu_drafts import _check as check_drafts
from tests.test_gpu_drafts import _make
from tests.test_gpu_w4 import _check as check_product
from tests.test_gpu_w4 import _weights, _x

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch", [1, 7, 30, 70])  # clusters of 8, 8, 4 and 2
@pytest.mark.parametrize("with_draft", [True, False])
def test_sequences_that_draw_and_sequences_that_do_not(batch, with_draft):
    """Greedy ones, ones that end at a row without a distribution, empty ones and ones that draw, of lengths that are no multiple of a warp."""
    rows = [[37, 0, 5, 1][b % 4] for b in range(batch)]
    m = _make(rows, 40000, torch.float32, with_draft, [[0.0, 1.0, 0.8, 0.0, 1.0][b % 5] for b in range(batch)])
    m["ua"].zero_()  # all accepted up to there
    bad = [b for b in range(batch) if b % 3 == 2 and rows[b] > 1]
    for b in bad:
        m["target"][m["cu"][b] + 3, 39999] = float("nan")
    check_drafts(m, vb.DEV_LOGITS if any(m["temps"][b] > 0 for b in bad) else 0)


@pytest.mark.parametrize("rows,n,k", [(9, 72, 4096), (13, 136, 8192), (33, 200, 16384), (61, 8, 8192)])
def test_slices_of_outputs_that_fill_no_tile(rows, n, k):
    _, w4 = _weights(n, k, 128)
    for dtype in (torch.float32, torch.bfloat16):
        check_product(_x(rows, k), w4, dtype, residual=torch.randn(rows, n, device="cuda:0"))
