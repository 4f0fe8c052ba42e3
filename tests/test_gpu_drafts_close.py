"""Drafts that nearly agree with the target: what is drawn from max(0, p - q) against 64 bits, p and q closer than fp32 tells apart."""
import math

import pytest
import torch

from paper_2509_24257_b200 import binding as vb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ONE = 1.0 - 2.0 ** -24
# Of sums of p = 1: an exponential in 64 bits is off by less than 2^-38 (4e-12), p and q by two of them, running sums and the point by both together.
TOL = 4 * 4e-12


def _probs(rows, temp):
    x = rows.double()
    e = torch.exp((x - x.amax(-1, keepdim=True)) / temp)
    return e / e.sum(-1, keepdim=True)


def _draw(target, draft, x, us, temp=1.0):
    """One sequence per row of target, its drafted token x[row] rejected; the tokens drawn."""
    batch, vocab = target.shape
    rows = torch.arange(batch, device=DEV)
    full_t, full_d = [torch.stack([m, torch.zeros_like(m)], 1).reshape(2 * batch, vocab) for m in (target, draft)]
    tokens = torch.zeros(2 * batch, dtype=torch.int32, device=DEV)
    tokens[1::2] = x.to(torch.int32)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    rep = vb.verify_drafts(full_t, tokens, torch.arange(0, 2 * batch + 1, 2, dtype=torch.int32, device=DEV), 2,
                           torch.full((2 * batch,), ONE, device=DEV), us, draft=full_d,
                           temperature=torch.full((batch,), temp, dtype=torch.float32, device=DEV), status=status)
    assert int(status.item()) == 0 and rep.n_emitted.tolist() == [1] * batch
    got = rep.tokens[::2].long()
    assert bool((got >= 0).all())
    logp = _probs(target, temp)[rows, got].log()
    assert bool(((rep.logp[::2].double() - logp).abs() <= 2.0 ** -20 * (1 + logp.abs()) + 2.0 ** -22 * 20).all())
    return got


def _check_draws(target, draft, us, temp=1.0):
    temp = float(torch.tensor(temp, dtype=torch.float32))
    p, q = _probs(target, temp), _probs(draft, temp)
    x = torch.where(p > 0, q / p, 0.0).argmax(-1)
    rows = torch.arange(p.shape[0], device=DEV)
    assert bool((ONE * q[rows, x] > p[rows, x] * (1 + 1e-11)).all())  # rejected whatever the rounding
    got = _draw(target, draft, x, us, temp)
    left = (p - q).clamp_min(0.0)
    run = left.cumsum(-1)
    point = us.double() * run[:, -1]
    after, own = run[rows, got], left[rows, got]
    assert bool((p[rows, got] > q[rows, got] * (1 - 1e-11)).all())
    assert bool((after - own <= point + TOL).all())  # begins at or before the point
    assert bool((after > point - TOL).all())         # and ends behind it
    return got


def _numbers(n, g):
    us = torch.rand(n, generator=g, device=DEV)
    us[:2] = torch.tensor([0.0, ONE], device=DEV)[:n]
    return us


@pytest.mark.parametrize("noise", [0.3, 1e-2, 1e-3, 1e-4, 1e-5, 1e-6])
@pytest.mark.parametrize("batch,vocab", [(100, 300), (64, 5000), (3, 32000), (64, 32000), (90, 32000), (17, 128256)])
def test_drafts_that_differ_by_little(batch, vocab, noise):
    g = torch.Generator(device=DEV).manual_seed(batch + vocab)
    target = torch.randn(batch, vocab, generator=g, device=DEV) * 2.5
    draft = target + noise * torch.randn(batch, vocab, generator=g, device=DEV)
    for _ in range(3):
        _check_draws(target, draft, _numbers(batch, g))
    _check_draws(target, draft, _numbers(batch, g), 0.6)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,vocab", [(90, 700), (8, 32000), (40, 100003)])
def test_a_token_that_the_draft_lacks_is_what_is_drawn(batch, vocab, dtype):
    """Equal logits but for one that the draft masks: everything else is a little likelier in the draft."""
    g = torch.Generator(device=DEV).manual_seed(vocab)
    target = (torch.randn(batch, vocab, generator=g, device=DEV) * 1.5).to(dtype)
    rows = torch.arange(batch, device=DEV)
    best = target.float().argmax(-1)
    gone = torch.randint(0, vocab, (batch,), generator=g, device=DEV)
    gone = torch.where(gone == best, (gone + 1) % vocab, gone)
    draft = target.clone()
    draft[rows, gone] = -math.inf
    p, q = _probs(target, 1.0), _probs(draft, 1.0)
    keep = ONE * q[rows, best] > p[rows, best] * (1 + 1e-11)  # (the number next to one is not enough to reject where the masked one is rarer than 2^-24)
    assert int(keep.sum()) > batch // 2
    got = _draw(target[keep], draft[keep], best[keep], _numbers(int(keep.sum()), g))
    assert torch.equal(got, gone[keep])


@pytest.mark.parametrize("raise_by", [1e-2, 1e-4, 4e-6])
@pytest.mark.parametrize("batch,vocab", [(90, 700), (8, 32000), (33, 128256)])
def test_one_raised_token_leaves_the_others_in_proportion(batch, vocab, raise_by):
    """A draft with one logit a little larger: all others are a little likelier in the target, by the same factor."""
    g = torch.Generator(device=DEV).manual_seed(vocab + 1)
    target = torch.randn(batch, vocab, generator=g, device=DEV) * 1.5
    rows = torch.arange(batch, device=DEV)
    raised = torch.randint(0, vocab, (batch,), generator=g, device=DEV)
    target[rows, raised] = 1.0
    draft = target.clone()
    draft[rows, raised] = 1.0 + raise_by
    for _ in range(3):
        got = _check_draws(target, draft, _numbers(batch, g))
        assert not bool((got == raised).any())


@pytest.mark.parametrize("batch,vocab", [(5, 20000), (80, 900)])
def test_differences_confined_to_a_few_tokens(batch, vocab):
    """Two tokens swap a little probability; what the others differ by comes from rounding the logits alone, and they share one of many ties."""
    g = torch.Generator(device=DEV).manual_seed(vocab + 2)
    target = torch.randn(batch, vocab, generator=g, device=DEV).mul(8).round().div(8)
    draft = target.clone()
    target[:, 11], draft[:, 11] = 3.0, 3.0 - 3e-5
    target[:, vocab - 5], draft[:, vocab - 5] = 3.0, 3.0 + 3e-5
    us = _numbers(batch, g)
    got = _check_draws(target, draft, us)
    # the second takes what the first loses, and 2^-32 of p of the others change sides either way
    assert int((got == 11).sum()) >= batch - 2
