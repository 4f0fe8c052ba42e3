"""Attention over the paged cache where the sizes of its numbers lie far apart (needs a B200)."""
import pytest
import torch

from paper_2509_24257_b200 import binding as vb
from tests.paged_cases import Case, assert_within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, E4M3, INT8 = torch.bfloat16, torch.float8_e4m3fn, torch.int8
DTYPES = [BF16, E4M3, INT8]


def _set(c, t, b, p, value, col=slice(None)):
    """Entry `col` of all kv heads at position p of sequence b, in float32 pools."""
    t[int(c.table[b, p // c.ps]), :, p % c.ps, col] = value


def _floats(c):
    return (t.float() if c.dtype == BF16 else t.float() * s[..., None] for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)))


# first sequence: rows, positions; others behind it
GAPS = [
    ("one CTA", [1], [100]),
    ("one CTA, drafted rows", [3, 2], [200, 40]),
    ("few pieces", [1, 2], [700, 900]),
    ("many pieces", [2], [9000]),
    ("many rows", [20] * 160, [90] * 160),
    ("many rows, split", [40, 30], [2000, 1500]),
    ("one block of many rows", [16], [16000]),
]


# (an 8-bit vector with an infinite entry is NaN altogether; infinities in large calls: see the next test)
NON_FINITE = [(g, d, x) for g in GAPS for d in DTYPES for x in (float("nan"), float("inf"), -float("inf"))
              if x != x or d == BF16 and g in GAPS[:4]]


@pytest.mark.parametrize("gap,dtype,value", NON_FINITE, ids=[f"{g[0]}, {d}, {x}" for g, d, x in NON_FINITE])
def test_a_value_that_is_not_finite_reaches_every_row_that_sees_it(gap, dtype, value):
    """One key scores 226 above the others, so that the others' weights vanish in float32: a NaN or infinite value among the
    others still makes the rows that see it NaN or infinite, wherever the two lie: in one warp's 16 keys, in two warps' of
    one tile, in two tiles or two CTAs, the large score before and behind."""
    name, rows, kv = gap
    heads, kv_heads = (8, 1) if name == "one block of many rows" else (8, 2)
    first = kv[0] - rows[0]  # visible to all rows of sequence 0
    for odd, top in ((3, 9), (9, 3), (3, 20), (20, 3), (5, 70), (70, 5), (2, first - 1), (first - 1, 2)):
        c = Case(dtype, heads, kv_heads, 128, 16, rows, kv, seed=41)
        u = torch.where(torch.rand(128, generator=torch.Generator().manual_seed(6)) < 0.5, -1.0, 1.0)
        c.q[:] = u.repeat(heads).to(BF16)
        k, v = _floats(c)
        _set(c, k, 0, top, 20.0 * u)  # scores 20 * 128 / sqrt(128)
        _set(c, v, 0, odd, value, 7)
        c.set_pools(k.to(BF16), v.to(BF16))
        cache, r = c.device()
        got = vb.op_attention_paged(c.dq, cache, r)
        r.check()
        n = rows[0]
        if len(rows) > 8:  # the others are there to make the call large
            c.rows, c.kv = c.rows[:1], c.kv[:1]
        ref, tol, _, _ = c.attention()
        assert not bool(ref[:n, :, 7].isfinite().any())
        used = int(c.cu[len(c.rows)])
        assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used], f"{odd} {top}")


@pytest.mark.parametrize("name,rows,kv", GAPS[4:], ids=[g[0] for g in GAPS[4:]])
def test_an_infinite_value_of_a_vanishing_weight_in_a_large_call_is_not_lost(name, rows, kv):
    """The kernel of many rows multiplies weights that vanished: infinity or NaN in the columns, nothing elsewhere."""
    heads, kv_heads = (8, 1) if name == "one block of many rows" else (8, 2)
    first = kv[0] - rows[0]
    for odd, top in ((3, 9), (20, 3), (2, first - 1), (first - 1, 2)):
        c = Case(BF16, heads, kv_heads, 128, 16, rows, kv, seed=42)
        u = torch.where(torch.rand(128, generator=torch.Generator().manual_seed(6)) < 0.5, -1.0, 1.0)
        c.q[:] = u.repeat(heads).to(BF16)
        k, v = _floats(c)
        _set(c, k, 0, top, 20.0 * u)
        _set(c, v, 0, odd, float("inf"), 7)
        c.set_pools(k.to(BF16), v.to(BF16))
        cache, r = c.device()
        got = vb.op_attention_paged(c.dq, cache, r)[:rows[0]].reshape(rows[0], heads, 128).isfinite().cpu()
        assert not bool(got[..., 7].any()) and bool(got[..., :7].all()) and bool(got[..., 8:].all()), (odd, top)


@pytest.mark.parametrize("rows,kv", [([3, 2], [200, 40]), ([4, 1], [900, 2000]), ([20] * 160, [90] * 160), ([40, 30], [2000, 1500])])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_later_token_of_great_size_does_not_disturb_the_rows_before_it(dtype, rows, kv):
    """The last token's key and value are 2^16 times as large as the others'.  Rows that may not see it give what they give
    without it: 8-bit operands are scaled to the largest of their reach, here 2^18 above the smallest, which leaves a scale
    within 2^-13 where the tolerance counts 2^-11 for the operand: a quarter more."""
    c = Case(dtype, 8, 2, 128, 16, rows, kv, seed=43)
    count = len(rows)
    if count > 8:
        c.rows, c.kv = c.rows[:2], c.kv[:2]
    ref, tol, _, _ = c.attention()
    c.rows, c.kv = list(rows), list(kv)
    k, v = _floats(c)
    for b in range(min(count, 2)):
        for t in (k, v):
            page, off = int(c.table[b, (kv[b] - 1) // c.ps]), (kv[b] - 1) % c.ps
            t[page, :, off] *= 2.0 ** 16
    c.set_pools(k.to(BF16), v.to(BF16))
    cache, r = c.device()
    got = vb.op_attention_paged(c.dq, cache, r)
    r.check()
    for b in range(min(count, 2)):
        at = slice(int(c.cu[b]), int(c.cu[b + 1]) - 1)
        assert_within(got[at].reshape(-1, c.H, c.dh), ref[at], 1.25 * tol[at], f"sequence {b}")
