"""Checking drafted tokens against the definition in 64 bits, one sequence at a time."""
import math

import pytest
import torch

from paper_2509_24257_b200 import binding as vb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _softmax(row, t):
    x = row.double()
    if t == 0:
        p = torch.zeros_like(x)
        p[int((x == x.max()).nonzero()[0])] = 1.0
        return p
    e = torch.exp((x - x.max()) / t)
    e[(x - x.max()) / t < -700] = 0.0
    return e / e.sum()


def _valid(row):
    return not bool(torch.isnan(row).any()) and bool(torch.isfinite(row.max()))


def _reference(target, tokens, cu, ua, us, draft, temps):
    """(emitted tokens, number emitted per sequence, log p) in plain Python over float64 rows on the CPU."""
    target, draft = target.float().cpu(), None if draft is None else draft.float().cpu()
    n = target.shape[0]
    out, logp, count = [-1] * n, [0.0] * n, []
    for b in range(len(cu) - 1):
        lo, hi, t = cu[b], cu[b + 1], temps[b]
        done = 0
        for r in range(lo, hi):
            more = r + 1 < hi
            if not _valid(target[r]) or (more and t > 0 and draft is not None and not _valid(draft[r])):
                break
            p = _softmax(target[r], t)
            res = p
            if more:
                x = tokens[r + 1]
                inside = 0 <= x < p.shape[0]
                q = torch.zeros_like(p)
                if draft is not None and t > 0:
                    q = _softmax(draft[r], t)
                elif inside:
                    q[x] = 1.0
                px = float(p[x]) if inside else 0.0
                if inside and ((px > 0) if t == 0 else ua[r + 1] * float(q[x]) < px):
                    out[r], logp[r] = x, math.log(px)
                    done += 1
                    continue
                if t > 0:
                    left = (p - q).clamp_min(0)
                    res = left if float(left.sum()) > 0 else p
            u = min(max(us[b], 0.0), 1.0) if us[b] == us[b] else 0.0
            run = torch.cumsum(res, 0)
            over = (run > u * run[-1]).nonzero()
            v = int(over[0]) if len(over) else int((res > 0).nonzero()[-1])
            out[r], logp[r] = v, math.log(float(p[v]))
            done += 1
            break
        count.append(done)
    return out, count, logp


def _make(rows, vocab, dtype, with_draft, temps, seed=0, spread=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = sum(rows)
    target = (torch.randn(n, vocab, generator=g, device=DEV) * spread).to(dtype)
    draft = (target.float() + 0.6 * torch.randn(n, vocab, generator=g, device=DEV)).to(dtype)
    cu = [sum(rows[:b]) for b in range(len(rows) + 1)]
    t = torch.tensor([temps[b] for b in range(len(rows)) for _ in range(rows[b])], device=DEV)
    noise = -torch.log(-torch.log(torch.rand(n, vocab, generator=g, device=DEV).clamp(1e-30, 1 - 1e-7)))
    picked = (draft.float() + noise * t[:, None] * (1.0 if with_draft else 0.3)).argmax(-1)
    tokens = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), picked[:-1]]).to(torch.int32) if n else torch.zeros(0, dtype=torch.int32, device=DEV)
    return dict(target=target, tokens=tokens, cu=cu, ua=torch.rand(n, generator=g, device=DEV), us=torch.rand(len(rows), generator=g, device=DEV),
                draft=draft if with_draft else None, temps=temps)


def _run(m, **kw):
    batch = len(m["cu"]) - 1
    max_rows = max([1] + [m["cu"][b + 1] - m["cu"][b] for b in range(batch)])
    kw.setdefault("kv_len", torch.full((batch,), 1000, dtype=torch.int32, device=DEV))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    rep = vb.verify_drafts(m["target"], m["tokens"], torch.tensor(m["cu"], dtype=torch.int32, device=DEV), max_rows, m["ua"], m["us"], draft=m["draft"],
                           temperature=torch.tensor(m["temps"], dtype=torch.float32, device=DEV), status=status, **kw)
    return rep, int(status.item())


def _check(m, want_status=0, **kw):
    rep, status = _run(m, **kw)
    temps = torch.tensor(m["temps"], dtype=torch.float32).tolist()
    out, count, logp = _reference(m["target"], m["tokens"].tolist(), m["cu"], m["ua"].tolist(), m["us"].tolist(), m["draft"], temps)
    assert rep.tokens.tolist() == out
    assert rep.n_emitted.tolist() == count
    assert rep.new_len.tolist() == [1000 - (m["cu"][b + 1] - m["cu"][b]) + c for b, c in enumerate(count)]
    # log p: a difference of fp32 logits over T (2^-22 of it), and the log of a sum of exp2.approx (2^-22 each) and its rounding
    for a, b in zip(rep.logp.tolist(), logp):
        assert abs(a - b) <= 2.0 ** -20 * (1 + abs(b)) + 2.0 ** -22 * 20
    assert status == want_status
    return rep


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("vocab", [1, 2, 7, 33, 100, 1000, 1023, 4097, 32000, 50257])
def test_vocabularies(vocab, with_draft, dtype):
    for seed in range(3):
        _check(_make([5, 1, 3, 2], vocab, dtype, with_draft, [1.0, 0.7, 0.0, 1.3], seed))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_vocabulary(dtype):
    _check(_make([6, 2, 9], 151936, dtype, True, [1.0, 0.5, 1.5]))
    _check(_make([4, 3], 128256, dtype, False, [1.0, 0.0]))


@pytest.mark.parametrize("vocab,dtype", [(50257, torch.float32), (100003, torch.bfloat16)])
def test_large_vocabulary_of_more_sequences_than_clusters_fit(vocab, dtype):
    _check(_make([2, 1] * 40, vocab, dtype, True, [0.9, 1.1] * 40))
    _check(_make([2, 1] * 40, vocab, dtype, False, [0.9, 1.1] * 40))


@pytest.mark.parametrize("rows", [[1], [0], [0, 0, 3], [1] * 40, [17, 0, 1], [64], [256], [3, 200, 2]])
def test_rows(rows):
    _check(_make(rows, 500, torch.float32, True, [0.8] * len(rows), spread=0.3))


def test_many_sequences():
    rows = [(i * 7) % 5 for i in range(700)]
    _check(_make(rows, 130, torch.float32, True, [[0.0, 0.6, 1.0][i % 3] for i in range(700)]))


@pytest.mark.parametrize("vocab", [400, 40000])
def test_far_temperatures_and_peaked_rows(vocab):
    m = _make([4] * 6, vocab, torch.float32, True, [1e-4, 0.02, 100.0, 1e20, 2.0 ** -100, 2.0 ** 100])
    _check(m)
    m = _make([3, 3], vocab, torch.bfloat16, False, [1.0, 1.0], spread=40.0)
    _check(m)


@pytest.mark.parametrize("vocab", [900, 30000])
def test_ties_of_large_logits_at_small_temperatures(vocab):
    m = _make([5] * 8, vocab, torch.float32, True, [2.0 ** -100, 2.0 ** -60, 1e-9, 1e-4] * 2)
    g = torch.Generator(device=DEV).manual_seed(3)
    for name in ("target", "draft"):
        m[name] = torch.where(torch.rand(40, vocab, generator=g, device=DEV) < 0.3, 12345.678, m[name])
    m["tokens"] = m["draft"].roll(1, 0).argmax(-1).to(torch.int32)
    _check(m)
    _check(dict(m, draft=None))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_drafts_close_to_the_target_far_from_zero(dtype):
    """Logits near 500 at T = 0.01: log p is a difference of numbers near 72000."""
    m = _make([3] * 40, 2000, torch.float32, True, [0.01] * 40, spread=0.02)
    g = torch.Generator(device=DEV).manual_seed(4)
    m["target"] = (m["target"] + (500 if dtype == torch.float32 else 0)).to(dtype)
    m["draft"] = (m["target"].float() + 0.002 * torch.randn(120, 2000, generator=g, device=DEV)).to(dtype)
    m["ua"] = 0.9 + 0.1 * m["ua"]
    _check(m)


def test_numbers_next_to_the_border_are_decided_in_64_bits():
    """accept_u set to p / q rounded to fp32 and its two neighbours: fp32 sums of 3000 terms cannot tell them apart."""
    m = _make([9] * 30, 3000, torch.float32, True, [0.9] * 30, spread=0.8)
    for r in range(sum([9] * 30) - 1):
        p, q = _softmax(m["target"][r].cpu(), float(torch.tensor(0.9))), _softmax(m["draft"][r].cpu(), float(torch.tensor(0.9)))
        x = int(m["tokens"][r + 1])
        u = torch.tensor(min(float(p[x] / q[x]), 1.0 - 2.0 ** -24), dtype=torch.float32)
        step = (r % 3) - 1
        m["ua"][r + 1] = torch.nextafter(u, torch.tensor(2.0 * step)) if step else u
    _check(m)
    m["draft"] = None
    for r in range(sum([9] * 30) - 1):
        m["ua"][r + 1] = float(_softmax(m["target"][r].cpu(), float(torch.tensor(0.9)))[int(m["tokens"][r + 1])])
    _check(m)


def test_draws_next_to_the_border():
    """sample_u just before and behind a border of the running sum (64-bit spacing is 10^9 times finer than fp32's steps of u)."""
    vocab = 20000
    m = _make([1] * 64, vocab, torch.float32, False, [1.0] * 64)
    for b in range(64):
        run = torch.cumsum(_softmax(m["target"][b].cpu(), 1.0), 0)
        u = torch.tensor(float(run[(b * 311) % vocab]), dtype=torch.float32)
        m["us"][b] = u if b % 2 else torch.nextafter(u, torch.tensor(2.0))
    _check(m)


def test_equal_distributions_accept_everything_below_one():
    m = _make([8] * 4, 1000, torch.bfloat16, True, [1.0] * 4)
    m["draft"] = m["target"].clone()
    m["ua"].fill_(1.0 - 2.0 ** -24)
    rep = _check(m)
    assert rep.n_emitted.tolist() == [8] * 4
    m["ua"].fill_(1.0)  # u q < p fails with p = q, and max(0, p - q) is empty: drawn from p
    _check(m)


def test_extreme_numbers():
    m = _make([5] * 8, 700, torch.float32, True, [1.0] * 8)
    for i, u in enumerate([0.0, -1.0, 1.0, 2.0, float("inf"), float("nan"), 1e-38, 1.0 - 2.0 ** -24]):
        m["ua"][5 * i:5 * i + 5] = u
        m["us"][i] = u
    _check(m)


def test_masked_entries_and_empty_residuals():
    m = _make([4] * 6, 900, torch.float32, True, [1.0, 0.5, 0.0] * 2)
    m["target"][:, ::3] = -math.inf
    m["draft"][:, 1::3] = -math.inf
    m["target"][5, :] = -math.inf
    m["target"][5, 17] = 3.0  # one token left
    m["target"][9:12, 100:] = torch.finfo(torch.float32).min
    _check(m)
    m["draft"] = None
    _check(m)


@pytest.mark.parametrize("vocab", [90, 5000])
@pytest.mark.parametrize("which", ["target", "draft"])
@pytest.mark.parametrize("bad", ["nan", "inf", "empty"])
def test_a_row_without_a_distribution_ends_its_sequence_only(which, bad, vocab):
    m = _make([5, 5, 5], vocab, torch.float32, True, [1.0, 1.0, 1.0])
    m["ua"].zero_()  # everything is accepted up to there
    if bad == "empty":
        m[which][7] = -math.inf
    else:
        m[which][7, vocab - 3] = float(bad)
    rep = _check(m, vb.DEV_LOGITS)
    assert rep.n_emitted.tolist() == [5, 2, 5]
    m["temps"] = [0.0] * 3
    _check(m, vb.DEV_LOGITS if which == "target" and rep.tokens is not None and _reaches(m, 7) else 0)


def _reaches(m, row):
    out, count, _ = _reference(m["target"], m["tokens"].tolist(), m["cu"], m["ua"].tolist(), m["us"].tolist(), m["draft"], m["temps"])
    b = max(b for b in range(len(count)) if m["cu"][b] <= row)
    return m["cu"][b] + count[b] == row


def test_temperatures_out_of_range():
    m = _make([3] * 6, 60, torch.float32, True, [1.0] * 6)
    m["temps"] = [-1.0, float("nan"), float("inf"), 1e-38, 1.0, 0.0]
    rep, status = _run(m)
    assert rep.n_emitted.tolist()[:4] == [0] * 4 and rep.tokens.tolist()[:12] == [-1] * 12 and status == vb.DEV_LOGITS
    assert rep.new_len.tolist()[:4] == [997] * 4
    good = dict(m, temps=[1.0] * 4 + [1.0, 0.0])
    want, _ = _run(good)
    assert rep.tokens.tolist()[12:] == want.tokens.tolist()[12:]


def test_tokens_outside_the_vocabulary_are_rejected():
    m = _make([4, 4, 4], 300, torch.float32, True, [1.0, 0.0, 1.0])
    m["ua"].zero_()
    m["tokens"][2], m["tokens"][5], m["tokens"][9] = 300, -5, 2 ** 31 - 1
    _check(m, vb.DEV_TOKEN_RANGE)
    m["draft"] = None
    _check(m, vb.DEV_TOKEN_RANGE)


def test_ties_go_to_the_lowest_index():
    m = _make([2, 2, 2], 5000, torch.bfloat16, False, [0.0] * 3)
    m["target"][:] = 1.5
    m["target"][2:4, 4000:] = 2.0
    m["target"][4:, 3:] = 2.0
    m["tokens"][:] = torch.tensor([0, 0, 0, 4000, 0, 4], dtype=torch.int32)
    rep = _check(m)
    assert rep.tokens.tolist() == [0, 0, 4000, 4000, 3, -1]


def test_strided_and_unaligned_rows_give_the_same():
    for dtype in (torch.bfloat16, torch.float32):
        m = _make([5, 3], 3001, dtype, True, [1.0, 0.8])
        want = _check(m)
        for off in (1, 3):
            wide = [torch.zeros(8, 3100, dtype=dtype, device=DEV) for _ in range(2)]
            for w, k in zip(wide, ("target", "draft")):
                w[:, off:off + 3001] = m[k]
            other = dict(m, target=wide[0][:, off:off + 3001], draft=wide[1][:, off:off + 3001])
            got = _check(other)
            assert got.tokens.tolist() == want.tokens.tolist()
        mixed = dict(m, draft=torch.cat([m["draft"], m["draft"][:, :6]], 1)[:, :3001])
        _check(mixed)


def test_rows_behind_the_last_sequence_and_bad_boundaries():
    m = _make([4, 4, 4], 200, torch.float32, True, [1.0] * 3)
    want, _ = _run(m)
    rep = vb.DraftReport(12, 2, DEV, True)
    rep.tokens.fill_(-7)
    rep.logp.fill_(-7)
    short = dict(m, cu=m["cu"][:3], us=m["us"][:2], temps=[1.0] * 2)
    got, status = _run(short, report=rep)
    assert got.tokens.tolist() == want.tokens.tolist()[:8] + [-7] * 4 and got.logp.tolist()[8:] == [-7.0] * 4 and status == 0
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for cu in ([0, 4, 400, 12], [0, -3, 4, 12], [4, 2, 8, 12], [0, 4, 12, 12]):
        status.zero_()
        r = vb.verify_drafts(m["target"], m["tokens"], torch.tensor(cu, dtype=torch.int32, device=DEV), 4, m["ua"], m["us"], draft=m["draft"], status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == vb.DEV_ROWS_RANGE and 0 in r.n_emitted.tolist()


def test_captured_on_another_stream_and_twice_at_once():
    m = _make([6] * 5, 8000, torch.bfloat16, True, [1.0] * 5)
    want, _ = _run(m)
    cu = torch.tensor(m["cu"], dtype=torch.int32, device=DEV)
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    reps = [vb.verify_drafts(m["target"], m["tokens"], cu, 6, m["ua"], m["us"], draft=m["draft"], stream=side[i % 2]) for i in range(8)]
    torch.cuda.synchronize()
    for r in reps:
        assert torch.equal(r.tokens, want.tokens) and torch.equal(r.n_emitted, want.n_emitted) and torch.equal(r.logp, want.logp)
    rep, ws = vb.DraftReport(30, 5, DEV, False), torch.empty(vb.verify_drafts_workspace(30), dtype=torch.uint8, device=DEV)
    us = m["us"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.verify_drafts(m["target"], m["tokens"], cu, 6, m["ua"], us, draft=m["draft"], report=rep, workspace=ws)
    us.copy_(m["us"].flip(0))
    graph.replay()
    torch.cuda.synchronize()
    other, _ = _run(dict(m, us=us))
    assert torch.equal(rep.tokens, other.tokens)


def test_what_is_emitted_is_distributed_like_the_target():
    """Draws over a grid of both numbers: the first emitted token's frequencies are p, whatever the draft (the point of the procedure)."""
    vocab, n = 6, 4096
    g = torch.Generator(device=DEV).manual_seed(5)
    t, d = torch.randn(vocab, generator=g, device=DEV), torch.randn(vocab, generator=g, device=DEV)
    q = torch.softmax(d.double(), 0)
    # drafted tokens in proportion to q, exactly spread numbers: (i + 1/2) / 64 for both
    seen = torch.zeros(vocab, dtype=torch.float64, device=DEV)
    grid = (torch.arange(64, device=DEV).float() + 0.5) / 64
    for x in range(vocab):
        target, draft = t.repeat(2 * n, 1), d.repeat(2 * n, 1)
        tokens = torch.full((2 * n,), x, dtype=torch.int32, device=DEV)
        ua = grid.repeat_interleave(64).repeat_interleave(2)
        rep = vb.verify_drafts(target, tokens, torch.arange(0, 2 * n + 1, 2, dtype=torch.int32, device=DEV), 2, ua, grid.repeat(64), draft=draft)
        seen += q[x] * torch.bincount(rep.tokens[::2].long(), minlength=vocab).double() / n
    # each of the two grids of 64 places a share to within 1 / 64
    assert bool(((seen - torch.softmax(t.double(), 0)).abs() < 2 / 64).all())


def test_refusals():
    m = _make([3, 2], 100, torch.float32, True, [1.0, 1.0])
    cu = torch.tensor(m["cu"], dtype=torch.int32, device=DEV)

    def call(**kw):
        a = dict(target=m["target"], tokens=m["tokens"], cu_rows=cu, max_rows=3, accept_u=m["ua"], sample_u=m["us"], draft=m["draft"])
        a.update(kw)
        return vb.verify_drafts(**a)

    for kw in (dict(target=m["target"].half()), dict(draft=m["draft"].to(torch.bfloat16)), dict(draft=m["draft"][:, :50]), dict(tokens=m["tokens"].long()),
               dict(tokens=m["tokens"][:3]), dict(accept_u=m["ua"].double()), dict(sample_u=m["us"][:1]), dict(cu_rows=cu.long()),
               dict(temperature=torch.ones(3, device=DEV)), dict(kv_len=torch.ones(2, device=DEV)), dict(status=torch.zeros(2, dtype=torch.int32, device=DEV)),
               dict(target=m["target"].cpu()), dict(workspace=torch.zeros(4, device=DEV))):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(vb.VerillmError):
        call(max_rows=257)
    with pytest.raises(vb.VerillmError):
        call(workspace=torch.zeros(64, dtype=torch.uint8, device=DEV))
