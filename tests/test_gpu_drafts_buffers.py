"""verify_drafts through its C entry over buffers that hold no more than the header asks for."""
import ctypes as C

import pytest
import torch

from paper_2509_24257_b200 import binding as vb
from tests.test_gpu_drafts import _make, _reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [130, 40000])
@pytest.mark.parametrize("rows", [[1], [4, 2, 5], [3] * 30 + [1]])
def test_draft_logits_end_before_the_last_row(rows, vocab, dtype):
    """The draft's buffer ends with the last row that a token follows (what lies behind it here is NaN); the last rows of other sequences are NaN too."""
    m = _make(rows, vocab, dtype, True, [0.9] * len(rows))
    cu, n = m["cu"], sum(rows)
    pool = torch.full((n * vocab,), float("nan"), dtype=dtype, device=DEV)
    draft = pool.view(n, vocab)
    for b in range(len(rows)):
        draft[cu[b]:cu[b + 1] - 1] = m["draft"][cu[b]:cu[b + 1] - 1]
    i32 = lambda k: torch.full((k,), -9, dtype=torch.int32, device=DEV)  # noqa: E731
    tokens, count, logp, status = i32(n), i32(len(rows)), torch.zeros(n, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    cu_dev, temp = torch.tensor(cu, dtype=torch.int32, device=DEV), torch.full((len(rows),), 0.9, device=DEV)
    ws = torch.empty(vb.verify_drafts_workspace(n), dtype=torch.uint8, device=DEV)
    d = vb.DraftsC(m["target"].data_ptr(), draft.data_ptr(), vocab, vocab, vb.F32 if dtype == torch.float32 else vb.BF16, vocab, len(rows), n, max(rows),
                   cu_dev.data_ptr(), m["tokens"].data_ptr(), None, temp.data_ptr(), m["ua"].data_ptr(), m["us"].data_ptr())
    r = vb.DraftReportC(tokens.data_ptr(), count.data_ptr(), logp.data_ptr(), None)
    torch.cuda.synchronize()
    assert vb.lib().verillm_verify_drafts(C.byref(d), C.byref(r), ws.data_ptr(), ws.numel(), status.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    want, counts, _ = _reference(m["target"], m["tokens"].tolist(), cu, m["ua"].tolist(), m["us"].tolist(), m["draft"], temp.tolist())
    assert tokens.tolist() == want and count.tolist() == counts and int(status.item()) == 0


@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("temp", [0.0, 1.0])
def test_a_last_row_without_a_distribution(with_draft, temp):
    """Everything is accepted up to the buffers' last row, which nothing follows and nothing can be drawn from."""
    m = _make([1, 4], 50000, torch.float32, with_draft, [temp] * 2)
    m["target"][[0, 4]] = float("nan")
    m["tokens"][2:] = m["target"][1:4].argmax(-1).to(torch.int32)
    m["ua"].zero_()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    rep = vb.verify_drafts(m["target"], m["tokens"], torch.tensor(m["cu"], dtype=torch.int32, device=DEV), 4, m["ua"], m["us"], draft=m["draft"],
                           temperature=torch.full((2,), temp, device=DEV), status=status)
    assert rep.tokens.tolist() == [-1] + m["tokens"].tolist()[2:] + [-1] and rep.n_emitted.tolist() == [0, 3]
    assert int(status.item()) == vb.DEV_LOGITS
