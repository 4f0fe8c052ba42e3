"""How exact each kernel of the paged attention is: the stated precision, not the loosest of the two (needs a B200)."""
import pytest
import torch

from paper_2509_24257_b200 import binding as vb
from tests.paged_cases import Case, assert_within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, E4M3, INT8 = torch.bfloat16, torch.float8_e4m3fn, torch.int8
DTYPES = [BF16, E4M3, INT8]
U, E = 2.0 ** -8, 2.0 ** -24  # half steps of bf16 and float32

FEW = [  # heads, kv heads, head_dim, page, rows, kv: at most 24 packed rows per sequence
    (16, 4, 64, 16, [1] * 5, [500, 1, 33, 250, 64]),
    (32, 8, 128, 16, [1] * 40, [90 + 7 * i for i in range(40)]),   # whole contexts and split ones
    (32, 8, 128, 64, [1, 1], [9000, 700]),                         # joined by many CTAs
    (32, 8, 128, 16, [5, 3, 6], [1500, 40, 333]),                  # three blocks of eight rows
    (12, 4, 64, 32, [4, 2], [900, 20]),                            # two
    (8, 1, 128, 16, [2, 1], [5000, 100]),
]
MANY = [
    (32, 8, 128, 16, [200, 33], [1000, 500]),
    (16, 4, 64, 64, [150, 90, 300], [700, 1200, 300]),
    (8, 1, 128, 64, [200], [3000]),
]


def _definition(c):
    """Per packed row and head in float64: out, sum p |v|, the largest score's sum |q k| / sqrt(dh), the sum |k| of the largest
    key, the largest |v|, the positions."""
    used, H, dh = int(c.cu[-1]), c.H, c.dh
    out, weight = torch.zeros(2, used, H, dh, dtype=torch.float64)
    size, ksum, vmax, length = torch.zeros(4, used, H, 1, dtype=torch.float64)
    for b, nb in enumerate(c.rows):
        k, v = c.positions(b)
        L, r0 = c.kv[b], int(c.cu[b])
        keep = torch.arange(L)[None, :] <= torch.arange(L - nb, L)[:, None]
        for h in range(H):
            kh, rows = h * c.KV // H, slice(r0, r0 + nb)
            q = c.q[rows, h * dh:(h + 1) * dh].double()
            p = torch.softmax(((q @ k[:, kh].T) / dh ** 0.5).masked_fill(~keep, -float("inf")), -1)
            out[rows, h], weight[rows, h] = p @ v[:, kh], p @ v[:, kh].abs()
            size[rows, h, 0] = (q.abs() @ k[:, kh].abs().T / dh ** 0.5).masked_fill(~keep, 0.0).amax(-1)
            ksum[rows, h] = q.abs().amax(-1, keepdim=True) * k[:, kh].abs().sum(-1).amax() / dh ** 0.5
            vmax[rows, h], length[rows, h] = v[:, kh].abs().max(), L
    return out, weight, size, ksum, vmax, length


def _relative(x, ref):
    return float((x.double().cpu() - ref).norm() / ref.norm())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", FEW)
def test_few_rows(shape, dtype):
    """bf16 pools: a probability enters as two bf16 numbers, the second the remainder of the first: off by 2^-16 at most.
    8-bit pools: codes are exact, key scales multiply scores in float32, a probability times its value's scale is rounded to
    fp16: 2^-11, or for each key 2^-31 of the largest value where the probabilities sum to 1 or more; a query entry below
    2^-14 of its row's largest is off by 2^-25 of that.  A score is a float32 sum of dh products with up to three factors,
    exp2 adds 2^-21, sums over L keys (L + 64) 2^-24, the output is rounded to bf16."""
    c = Case(dtype, *shape, seed=61, width_extra=0)
    cache, rows = c.device()
    got = vb.op_attention_paged(c.dq, cache, rows)[:int(c.cu[-1])].reshape(-1, c.H, c.dh)
    rows.check()
    out, weight, size, ksum, vmax, length = _definition(c)
    eight = dtype != BF16
    d = (c.dh + 4) * E * size + (2.0 ** -25 * ksum if eight else 0.0)
    inner = weight * ((2.0 ** -11 if eight else 2.0 ** -16) + 2 * d + 2.0 ** -21 + (length + 64) * E)
    inner = inner + (length * 2.0 ** -31 * vmax if eight else 0.0)
    assert_within(got, out, inner * (1 + U) + U * out.abs())
    # In the 2-norm: rounding the exact result to bf16 is off by R.  fp16 probabilities add independent errors eight times smaller
    # per key than a bf16 rounding's; over all entries the whole is within a tenth of R.
    assert _relative(got, out) <= 1.1 * _relative(out.to(BF16), out), (_relative(got, out), _relative(out.to(BF16), out))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", MANY)
def test_many_rows(shape, dtype):
    """bf16 pools: a probability is rounded to bf16, an independent error per key of the relative size of the output's own: over
    all entries sqrt(2) times R, 1.6 allowed.  8-bit pools: keys, values and probabilities are rounded to fp16, eight times finer."""
    c = Case(dtype, *shape, seed=62, width_extra=0)
    cache, rows = c.device()
    got = vb.op_attention_paged(c.dq, cache, rows)[:int(c.cu[-1])].reshape(-1, c.H, c.dh)
    rows.check()
    out = _definition(c)[0]
    most = 1.6 if dtype == BF16 else 1.2
    assert _relative(got, out) <= most * _relative(out.to(BF16), out), (_relative(got, out), _relative(out.to(BF16), out))


@pytest.mark.parametrize("out", [BF16, torch.float32])
@pytest.mark.parametrize("dtype", DTYPES)
def test_read_is_the_float32_product_bit_for_bit(dtype, out):
    """code * scale in float32, then the output's type: two roundings to nearest."""
    for shape in ((32, 8, 128, 16, [1] * 9, [1, 16, 17, 31, 32, 33, 500, 64, 2]), (8, 4, 64, 64, [130, 3], [200, 3])):
        c = Case(dtype, *shape, seed=63, pad=0)
        cache, rows = c.device()
        k, v = vb.kv_read(cache, rows, c.n, out)
        rows.check()
        for got, pool, scale in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
            for b, nb in enumerate(c.rows):
                pos = torch.arange(c.kv[b] - nb, c.kv[b])
                page = c.table[b][pos // c.ps].long()
                x = pool[page, :, pos % c.ps].float() if dtype != E4M3 else pool.view(torch.uint8)[page, :, pos % c.ps].view(E4M3).float()
                if scale is not None:
                    x = x * scale[page, :, pos % c.ps][..., None]
                want = x.to(out)
                at = int(c.cu[b])
                assert torch.equal(got[at:at + nb].cpu(), want), (b, float((got[at:at + nb].cpu().double() - want.double()).abs().max()))
