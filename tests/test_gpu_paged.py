"""The paged key/value cache on the device against its definition in float64 (needs a B200)."""
import numpy as np
import pytest
import torch

from paper_2509_24257_b200 import binding as vb
from tests.paged_cases import Case, assert_within, quantise

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, E4M3, INT8 = torch.bfloat16, torch.float8_e4m3fn, torch.int8
DTYPES = [BF16, E4M3, INT8]


def _bytes(t):
    return t.contiguous().view(torch.uint8).cpu()


# --------------------------------------------------------------------------- write and read

WRITES = [  # heads, kv heads, head_dim, page, rows, kv
    (4, 4, 64, 16, [1], [1]),
    (32, 8, 128, 16, [1] * 9, [1, 16, 17, 31, 32, 33, 500, 0, 2]),  # a row without a position (kv 0)
    (16, 4, 64, 32, [5, 0, 37, 64, 1], [5, 9, 40, 64, 300]),
    (8, 1, 128, 64, [130, 3], [200, 3]),
    (4, 2, 64, 256, [20, 7], [12, 300]),  # more rows than positions: the first 8 do not exist
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", WRITES)
def test_write_stores_the_definition_and_nothing_else(shape, dtype):
    c = Case(dtype, *shape, seed=3)
    cache, rows = c.device()
    vb.kv_write(cache, rows, c.dk_new, c.dv_new)
    rows.check()
    want = [t.clone() if t is not None else None for t in (c.k, c.v, c.k_scale, c.v_scale)]
    for b, n in enumerate(c.rows):
        for i in range(n):
            p = c.kv[b] - n + i
            if p < 0:
                continue
            page, off, r = int(c.table[b, p // c.ps]), p % c.ps, int(c.cu[b]) + i
            for j, x in enumerate((c.k_new, c.v_new)):
                x = x[r].reshape(c.KV, c.dh)
                if dtype == BF16:
                    want[j][page, :, off] = x
                else:
                    codes, scale = quantise(x.float(), dtype)
                    want[j].view(torch.uint8)[page, :, off] = codes.view(torch.uint8)
                    want[2 + j][page, :, off] = scale
    for got, ref, name in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), want, ("k", "v", "k_scale", "v_scale")):
        if ref is not None:
            assert int((_bytes(got) != _bytes(ref)).sum()) == 0, name


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", WRITES)
def test_read_returns_what_is_stored(shape, dtype, out):
    c = Case(dtype, *shape, seed=4)
    cache, rows = c.device()
    dst = tuple(torch.full((c.n, c.KV, c.dh), 7.0, dtype=out, device=DEV) for _ in range(2))
    got = vb.kv_read(cache, rows, c.n, out, out=dst)
    rows.check()
    ref = torch.full((2, c.n, c.KV, c.dh), 7.0, dtype=torch.float64)  # rows behind the last sequence keep their values
    for b, n in enumerate(c.rows):
        k, v = c.positions(b)
        for i in range(n):
            p = c.kv[b] - n + i
            ref[0, int(c.cu[b]) + i], ref[1, int(c.cu[b]) + i] = (k[p], v[p]) if p >= 0 else (0.0, 0.0)
    half = 2.0 ** -24 if out == torch.float32 else 2.0 ** -8 + 2.0 ** -24  # code * scale in float32, then the output's type
    for x, y in zip(got, ref):
        assert_within(x, y, y.abs() * (0.0 if dtype == BF16 else half))


@pytest.mark.parametrize("dtype", [E4M3, INT8])
def test_write_of_zero_tiny_huge_and_non_finite_vectors(dtype):
    c = Case(dtype, 2, 2, 64, 16, [12], [12], seed=5)
    x = c.qkv
    cols = slice(2 * 64, 6 * 64)  # k and v columns
    x[0, cols] = 0.0
    x[1, cols] = 2.0 ** -126
    x[2, cols] = -(2.0 ** -112)
    x[3, cols] = torch.finfo(torch.bfloat16).max
    x[4, cols] *= 1e30
    x[5, 2 * 64 + 3] = float("nan")   # key of head 0
    x[6, 4 * 64 + 5] = float("inf")   # value of head 0
    x[7, 3 * 64 + 63] = -float("inf")  # key of head 1
    cache, rows = c.device()
    vb.kv_write(cache, rows, c.dk_new, c.dv_new)
    k, v = vb.kv_read(cache, rows, c.n, torch.float32)
    for got, src, pool, scales in ((k, c.k_new, cache.k, cache.k_scale), (v, c.v_new, cache.v, cache.v_scale)):
        codes, scale = quantise(src[:12].reshape(12, 2, 64).float(), dtype)
        page = int(c.table[0, 0])
        assert torch.equal(_bytes(pool[page, :, :12].transpose(0, 1)), _bytes(codes))
        assert torch.equal(scales[page, :, :12].T.cpu().isnan(), scale.isnan())
        assert torch.equal(scales[page, :, :12].T.cpu().nan_to_num(-1.0), scale.nan_to_num(-1.0))
        ref = codes.double() * scale.double()[..., None]
        assert_within(got[:12], ref, ref.abs() * 2.0 ** -24)
    assert bool(k[5, 0].isnan().all()) and bool(k[5, 1].isfinite().all()) and bool(v[5].isfinite().all())
    assert bool(v[6, 0].isnan().all()) and bool(k[6].isfinite().all()) and bool(k[7, 1].isnan().all())


def test_quantisation_error_is_at_most_half_a_step():
    c = Case(E4M3, 4, 4, 128, 16, [64], [64], seed=6)
    for dtype in (E4M3, INT8):
        c.dtype = dtype
        c.set_pools(torch.zeros_like(c.k, dtype=BF16), torch.zeros_like(c.v, dtype=BF16))
        cache, rows = c.device()
        vb.kv_write(cache, rows, c.dk_new, c.dv_new)
        k, _ = vb.kv_read(cache, rows, c.n, torch.float32)
        x = c.k_new[:64].double().reshape(64, 4, 128)
        amax = x.abs().amax(-1, keepdim=True)
        # e4m3: half a step is 2^-4 of the value, or 2^-10 in code units below the smallest normal code; int8: half a
        # code unit; each with float32's roundings of the factor and the product
        half = torch.maximum(x.abs() * 2.0 ** -4, 2.0 ** -10 * amax / 448) if dtype == E4M3 else 0.5 * amax / 127
        assert bool(((k[:64].double().cpu() - x).abs() <= half * (1 + 2.0 ** -18) + amax * 2.0 ** -21).all())


# --------------------------------------------------------------------------- attention

ATTEND = [  # heads, kv heads, head_dim, page, rows, kv
    (4, 4, 64, 16, [1], [1]),
    (16, 4, 64, 16, [1], [500]),
    (32, 8, 128, 16, [1] * 7, [1, 15, 16, 17, 64, 65, 1000]),  # decode step, ends around page and tile borders
    (64, 8, 128, 64, [1, 1], [2100, 130]),                      # eight query heads share a kv head
    (32, 8, 128, 16, [3, 4, 1, 2], [3, 200, 129, 64]),          # drafted tokens, one sequence is only those
    (12, 4, 64, 32, [5, 1, 3], [70, 33, 3]),                    # three query heads per kv head
    (28, 4, 128, 32, [4, 2], [130, 300]),                       # seven
    (8, 8, 128, 128, [8, 7, 2], [8, 260, 129]),                 # no sharing
    (16, 4, 64, 32, [37, 0, 64, 1, 130], [37, 20, 300, 77, 130]),  # a mixture, one sequence without rows
    (32, 8, 128, 16, [100, 33], [100, 500]),
    (4, 2, 64, 256, [20, 7], [12, 300]),                        # more rows than positions: the first 8 attend to nothing
    (4, 2, 64, 16, [3, 2], [0, 1]),                             # nothing cached at all
    (2, 1, 128, 16, [1], [5000]),                               # one long sequence over many CTAs
    (8, 1, 128, 64, [200], [1500]),
    (32, 1, 64, 16, [3], [333]),                                # 32 query heads on one kv head
    (128, 1, 64, 32, [1, 5], [200, 100]),                       # 128: the most
    (4, 4, 128, 256, [260, 129], [1000, 129]),                  # many tokens per block, a page longer than a tile
    (14, 2, 64, 16, [300, 31, 2], [300, 2000, 513]),            # blocks that do not fill their rows
    (32, 8, 128, 64, [64], [8192]),                             # one block whose tiles lie in many CTAs
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", ATTEND)
def test_attention_matches_the_definition(shape, dtype):
    c = Case(dtype, *shape, seed=11)
    cache, rows = c.device()
    out = torch.full((c.n, c.H * c.dh + 16), 9.0, dtype=BF16, device=DEV)
    lse = torch.full((c.n, c.H), 9.0, device=DEV)
    vb.op_attention_paged(c.dq, cache, rows, out=out[:, :c.H * c.dh], lse=lse)
    rows.check()
    ref, tol, lref, ltol = c.attention()
    used = int(c.cu[-1])
    assert_within(out[:used, :c.H * c.dh].reshape(used, c.H, c.dh), ref[:used], tol[:used], "out")
    assert_within(lse[:used], lref[:used], ltol[:used], "lse")
    assert bool((out[used:] == 9.0).all()) and bool((out[:, c.H * c.dh:] == 9.0).all()) and bool((lse[used:] == 9.0).all())


@pytest.mark.parametrize("heads,kv_heads,dh,rows,kv", [
    (8, 1, 128, [3, 1, 4, 2], [9000, 20000, 5000, 100]),  # long contexts beside short ones: pieces joined by many CTAs and by few
    (12, 4, 64, [1, 8], [30011, 4099]),
    (32, 1, 64, [1], [16000]),                            # more pieces than a warp has lanes
])
@pytest.mark.parametrize("dtype", DTYPES)
def test_few_rows_over_long_contexts(dtype, heads, kv_heads, dh, rows, kv):
    c = Case(dtype, heads, kv_heads, dh, 64, rows, kv, seed=29)
    cache, rows_d = c.device()
    lse = torch.zeros(c.n, c.H, device=DEV)
    got = vb.op_attention_paged(c.dq, cache, rows_d, lse=lse)
    rows_d.check()
    ref, tol, lref, ltol = c.attention()
    used = int(c.cu[-1])
    assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used])
    assert_within(lse[:used], lref[:used], ltol[:used], "lse")
    assert torch.equal(got[:used], vb.op_attention_paged(c.dq, cache, rows_d)[:used])


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_over_many_sequences(dtype):
    """More sequences than a CTA has threads: the share of each CTA is found in several passes."""
    rng = np.random.default_rng(5)
    kv = rng.integers(0, 90, size=300)
    rows = np.minimum(rng.integers(0, 3, size=300), 2)
    c = Case(dtype, 4, 2, 64, 16, rows.tolist(), kv.tolist(), seed=12)
    cache, rows_d = c.device()
    got = vb.op_attention_paged(c.dq, cache, rows_d)
    rows_d.check()
    ref, tol, _, _ = c.attention()
    used = int(c.cu[-1])
    assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used])


@pytest.mark.parametrize("dtype", DTYPES)
def test_more_sequences_than_the_kernels_keep_at_hand(dtype):
    """1100 sequences: beyond the boundaries that write and read keep in shared memory, and beyond the threads of both
    attention kernels.  Written, read back and attended to, with and without a long chunk among the rows."""
    rng = np.random.default_rng(9)
    kv = rng.integers(1, 60, size=1100)
    for most in (2, 40):
        rows = np.minimum(rng.integers(0, 3, size=1100), kv)
        kv[700], rows[700] = 59, min(most, 59)
        c = Case(dtype, 4, 2, 64, 16, rows.tolist(), kv.tolist(), seed=22)
        cache, rows_d = c.device()
        vb.kv_write(cache, rows_d, c.dk_new, c.dv_new)
        k, v = vb.kv_read(cache, rows_d, c.n, torch.float32)
        used = int(c.cu[-1])
        for got, src in ((k, c.k_new), (v, c.v_new)):
            x = src[:used].float().reshape(used, 2, 64)
            if dtype != BF16:
                codes, scale = quantise(x, dtype)
                x = codes.float() * scale[..., None]
            assert torch.equal(got[:used].cpu(), x)
        c.k, c.v = cache.k.cpu(), cache.v.cpu()
        c.k_scale, c.v_scale = (None, None) if dtype == BF16 else (cache.k_scale.cpu(), cache.v_scale.cpu())
        got = vb.op_attention_paged(c.dq, cache, rows_d)
        rows_d.check()
        ref, tol, _, _ = c.attention()
        assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used])


def test_workspace_of_a_larger_call_serves_smaller_ones():
    c = Case(INT8, 8, 2, 128, 16, [40], [600], seed=23)
    cache, r = c.device()
    needs = [vb.attention_paged_workspace(cache, r, n, 8) for n in range(1, 41)]
    assert all(a <= b for a, b in zip(needs, needs[1:]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,kv_heads,dh,page,batch,most_rows,most_kv", [
    (16, 8, 64, 16, 40, 300, 500),     # several blocks per CTA, many with one group of rows only
    (16, 4, 128, 32, 24, 70, 1600),    # many tiles per CTA
    (64, 8, 128, 64, 12, 100, 900),
    (28, 4, 64, 32, 30, 90, 300),      # 7 query heads per kv head: blocks of 224 rows
    (4, 4, 128, 16, 60, 400, 450),     # blocks of one and of two groups in turn
    (32, 8, 128, 16, 20, 24, 2500),    # up to 96 rows per block: both groups on the same rows
    (16, 2, 64, 64, 50, 16, 400),      # the same with few tiles, one in many cases
])
def test_chunks_of_a_large_batch(heads, kv_heads, dh, page, batch, most_rows, most_kv, dtype):
    rng = np.random.default_rng(7)
    kv = rng.integers(most_kv // 3, most_kv + 1, size=batch)
    rows = np.minimum(rng.integers(1, most_rows + 1, size=batch), kv)
    rows[0] = most_rows
    c = Case(dtype, heads, kv_heads, dh, page, rows.tolist(), kv.tolist(), seed=21)
    cache, rows_d = c.device()
    got = vb.op_attention_paged(c.dq, cache, rows_d)
    rows_d.check()
    ref, tol, _, _ = c.attention()
    used = int(c.cu[-1])
    assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used])


@pytest.mark.parametrize("rows,kv", [([1, 2], [100, 40]), ([6, 40], [100, 40])])
@pytest.mark.parametrize("dtype", DTYPES)
def test_non_finite_entries_reach_exactly_the_rows_that_see_them(dtype, rows, kv):
    """An infinite or NaN value (or key) of a late token must not leak into the rows before it."""
    c = Case(dtype, 8, 2, 128, 16, rows, kv, seed=13)
    k, v = (torch.zeros_like(t, dtype=torch.float32) for t in (c.k, c.v))
    g = torch.Generator().manual_seed(1)
    k.copy_(torch.randn(k.shape, generator=g))
    v.copy_(torch.randn(v.shape, generator=g))

    def at(b, p):
        return int(c.table[b, p // c.ps]), p % c.ps

    pg, off = at(0, 99)
    v[pg, 0, off, 5] = float("nan")      # last token of sequence 0, kv head 0
    pg, off = at(1, 38)
    v[pg, 1, off, 100] = float("inf")    # next to last token of sequence 1, kv head 1
    pg, off = at(1, 39)
    k[pg, 0, off, 0] = float("nan")      # last token of sequence 1, kv head 0
    c.set_pools(k.to(BF16), v.to(BF16))
    cache, rows_d = c.device()
    got = vb.op_attention_paged(c.dq, cache, rows_d)
    ref, tol, _, _ = c.attention()
    used = int(c.cu[-1])
    assert not bool(ref[:used].isfinite().all()) and bool(ref[:used].isfinite().any())
    assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used])


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_scores_and_a_late_maximum(dtype):
    """Scores of several hundred whose maximum keeps growing along the sequence: the reference is raised many times."""
    c = Case(dtype, 4, 2, 64, 16, [2, 20], [700, 400], seed=14)
    k, v = (t.float() if dtype == BF16 else t.float() * s[..., None] for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    for b in range(2):
        for p in range(c.kv[b]):
            k[int(c.table[b, p // 16]), :, p % 16] *= 0.02 * p
    c.set_pools(k.to(BF16), v.to(BF16))
    cache, rows = c.device()
    got = vb.op_attention_paged(c.dq, cache, rows)
    ref, tol, _, _ = c.attention()
    used = int(c.cu[-1])
    assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used])


@pytest.mark.parametrize("rows,kv", [([1, 2], [100, 40]), ([6, 40], [300, 140])])
@pytest.mark.parametrize("q_size,k_size", [(0.0, 1e-6), (0.0, 0.0), (1e-30, 1e-3), (1e25, 1e-25), (1e-25, 1e25)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_very_small_and_large_queries_and_keys(dtype, q_size, k_size, rows, kv):
    """Queries of zero over small keys (every visible key weighs the same), and sizes that only their product makes moderate."""
    c = Case(dtype, 8, 2, 128, 16, rows, kv, seed=24)
    k, v = (torch.zeros_like(t, dtype=torch.float32) for t in (c.k, c.v))
    g = torch.Generator().manual_seed(2)
    k.copy_(torch.randn(k.shape, generator=g) * k_size)
    v.copy_(torch.randn(v.shape, generator=g))
    c.set_pools(k.to(BF16), v.to(BF16))
    c.q.copy_(c.q.float() * q_size)
    cache, rows_d = c.device()
    lse = torch.zeros(c.n, c.H, device=DEV)
    got = vb.op_attention_paged(c.dq, cache, rows_d, lse=lse)
    rows_d.check()
    ref, tol, lref, ltol = c.attention()
    used = int(c.cu[-1])
    assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used])
    assert_within(lse[:used], lref[:used], ltol[:used], "lse")


def test_attention_agrees_with_the_packed_operator():
    """Whole sequences written into a bf16 cache and attended to from all their rows are op_attention."""
    lens, H, KV, dh = [130, 1, 257, 64], 32, 8, 128
    c = Case(BF16, H, KV, dh, 16, lens, lens, seed=15, pad=0, strided=False)
    cache, rows = c.device()
    vb.kv_write(cache, rows, c.dk_new, c.dv_new)
    got = vb.op_attention_paged(c.dq, cache, rows)
    want = vb.op_attention(c.qkv.to(DEV), c.cu, H, KV, dh)
    # both are within 2 * 2^-8 of sum p |v| + 2^-8 |out| of the exact value, and |v| < 6 here
    assert float((got.float() - want.float()).abs().max()) <= 4 * 2.0 ** -8 * 6


# --------------------------------------------------------------------------- in use


def test_a_decode_loop_writes_then_attends():
    """Prompts in one chunk, then eight decode steps of all sequences, write before attention, in one captured
    graph per step form: the outputs are those of the definition over the cache as it stands after each step."""
    prompts, H, KV, dh, ps = [40, 3, 17], 8, 2, 64, 16
    for dtype in DTYPES:
        total = [p + 8 for p in prompts]
        whole = Case(dtype, H, KV, dh, ps, total, total, seed=16, pad=0)
        whole.device()
        cache = vb.KVCache.alloc(whole.k.shape[0], ps, KV, dh, dtype)
        table = whole.table.to(DEV)
        q, k, v = whole.dq, whole.dk_new, whole.dv_new
        first = [int(x) for x in whole.cu[:-1]]

        def gather(x, spans):
            return torch.cat([x[first[b] + s:first[b] + e] for b, (s, e) in enumerate(spans)]).contiguous()

        outs = {}
        cu = torch.tensor(np.concatenate([[0], np.cumsum(prompts)]), dtype=torch.int32, device=DEV)
        rows = vb.PagedRows(table, cu, torch.tensor(prompts, dtype=torch.int32, device=DEV), max(prompts))
        spans = [(0, p) for p in prompts]
        vb.kv_write(cache, rows, gather(k, spans), gather(v, spans))
        outs["prompt"] = vb.op_attention_paged(gather(q, spans), cache, rows)
        # the step's buffers are fixed, so one captured graph serves all steps
        sq, sk, sv = (torch.zeros(3, x.shape[1], dtype=BF16, device=DEV) for x in (q, k, v))
        kv_len = torch.tensor(prompts, dtype=torch.int32, device=DEV)
        step_rows = vb.PagedRows(table, torch.arange(4, dtype=torch.int32, device=DEV), kv_len, 1)
        graph, so = torch.cuda.CUDAGraph(), torch.zeros(3, H * dh, dtype=BF16, device=DEV)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            kv_len.add_(1)
            vb.kv_write(cache, step_rows, sk, sv)
            vb.op_attention_paged(sq, cache, step_rows, out=so)
        for t in range(8):
            spans = [(p + t, p + t + 1) for p in prompts]
            for dst, src in ((sq, q), (sk, k), (sv, v)):
                dst.copy_(gather(src, spans))
            graph.replay()
            outs[t] = so.clone()
        # the definition over the finished cache: causality makes a row's result the same as at its own step
        whole.k, whole.v = cache.k.cpu(), cache.v.cpu()
        whole.k_scale, whole.v_scale = (None, None) if dtype == BF16 else (cache.k_scale.cpu(), cache.v_scale.cpu())
        ref, tol, _, _ = whole.attention()
        for key, got in outs.items():
            spans = [(0, p) for p in prompts] if key == "prompt" else [(p + key, p + key + 1) for p in prompts]
            assert_within(got.reshape(-1, H, dh), gather(ref, spans), gather(tol, spans), f"{dtype} {key}")


def test_shared_pages_and_repeated_calls_are_bit_equal():
    """Two sequences with the same first pages; a call repeated, on another stream, and with the caller's workspace
    gives the same bits."""
    for rows in ([1, 1], [40, 40]):
        c = Case(E4M3, 32, 8, 128, 16, rows, [1000, 1000], seed=17, pad=0)
        c.table[1, :30] = c.table[0, :30]
        cache, r = c.device()
        a = vb.op_attention_paged(c.dq, cache, r)
        ref, tol, _, _ = c.attention()
        assert_within(a.reshape(-1, 32, 128), ref, tol)
        ws = torch.empty(vb.attention_paged_workspace(cache, r, c.n, 32), dtype=torch.uint8, device=DEV)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        b = vb.op_attention_paged(c.dq, cache, r, stream=side, workspace=ws)
        b2 = vb.op_attention_paged(c.dq, cache, r, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and torch.equal(a, b2)


@pytest.mark.parametrize("rows", [[1, 1], [50, 50]])
def test_problems_only_the_device_sees_are_reported(rows):
    c = Case(INT8, 4, 2, 64, 16, rows, [64, 64], seed=18)
    cache, r = c.device()
    out = torch.zeros(c.n, 4 * 64, dtype=BF16, device=DEV)

    def status_of(call):
        r.status.zero_()
        call()
        return int(r.status.item())

    calls = [lambda: vb.kv_write(cache, r, c.dk_new, c.dv_new), lambda: vb.kv_read(cache, r, c.n, torch.float32),
             lambda: vb.op_attention_paged(c.dq, cache, r, out=out)]
    good = r.page_table.clone()
    for bad in (cache.n_pages, -1, 1 << 30):
        r.page_table[1, 3] = bad
        for call in calls:
            assert status_of(call) == vb.DEV_PAGE_RANGE
    with pytest.raises(RuntimeError):
        r.check()
    r.page_table.copy_(good)
    c.k, c.v, c.k_scale, c.v_scale = (t.cpu() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale))  # the writes above
    ref, tol, _, _ = c.attention()
    first = rows[0]
    for kv_len in ([64, -3], [64, 1 << 30]):  # the first sequence's results are not touched by the second's trouble
        r.kv_len.copy_(torch.tensor(kv_len, dtype=torch.int32))
        r.page_table.clamp_(0, cache.n_pages - 1)
        assert status_of(calls[2]) == vb.DEV_ROWS_RANGE
        assert_within(out[:first].reshape(first, 4, 64), ref[:first], tol[:first])
    r.kv_len.copy_(torch.tensor([64, 64], dtype=torch.int32))
    few = vb.PagedRows(r.page_table, r.cu_rows, r.kv_len, max_rows=1, status=r.status)
    if rows[0] > 1:
        out.fill_(9.0)
        assert status_of(lambda: vb.op_attention_paged(c.dq, cache, few, out=out)) == vb.DEV_ROWS_RANGE
        assert bool((out == 9.0).all())
    r.cu_rows.copy_(torch.tensor([0, rows[0], c.n + 5], dtype=torch.int32))
    for call in calls:
        assert status_of(call) == vb.DEV_ROWS_RANGE


def test_empty_calls_do_nothing():
    c = Case(E4M3, 4, 2, 64, 16, [2], [20], seed=19)
    cache, rows = c.device()
    before = cache.k.view(torch.uint8).clone()
    vb.kv_write(cache, rows, c.dk_new[:0], c.dv_new[:0])
    k, v = vb.kv_read(cache, rows, 0)
    assert k.shape == (0, 2, 64) and v.shape == (0, 2, 64)
    assert vb.op_attention_paged(c.dq[:0], cache, rows).shape == (0, 256)
    assert torch.equal(before, cache.k.view(torch.uint8))
    none = vb.PagedRows(rows.page_table, torch.zeros(2, dtype=torch.int32, device=DEV), rows.kv_len, 1, rows.status)
    out = torch.full((c.n, 256), 9.0, dtype=BF16, device=DEV)
    vb.op_attention_paged(c.dq, cache, none, out=out)  # all rows are padding
    rows.check()
    assert bool((out == 9.0).all())


def test_wrapper_refuses_what_the_kernels_cannot_take():
    c = Case(E4M3, 4, 2, 64, 16, [2], [20], seed=20)
    cache, rows = c.device()
    with pytest.raises(ValueError):
        vb.KVCache(cache.k, cache.v)  # no scales
    with pytest.raises(ValueError):
        vb.KVCache(cache.k.float(), cache.v.float())
    with pytest.raises(ValueError):
        vb.KVCache(cache.k[:, :, ::2], cache.v[:, :, ::2], cache.k_scale[:, :, ::2], cache.v_scale[:, :, ::2])
    with pytest.raises(ValueError):
        vb.PagedRows(rows.page_table.long(), rows.cu_rows, rows.kv_len, 2)
    with pytest.raises(ValueError):
        vb.PagedRows(rows.page_table, rows.cu_rows[:1], rows.kv_len, 2)
    with pytest.raises(ValueError):
        vb.op_attention_paged(c.dq.float(), cache, rows)
    with pytest.raises(ValueError):
        vb.op_attention_paged(c.dq.T.contiguous().T, cache, rows)
    with pytest.raises(ValueError):
        vb.kv_write(cache, rows, c.dk_new[:, :64], c.dv_new[:, :64])
    with pytest.raises(ValueError):
        vb.kv_read(cache, rows, 2, torch.float16)
    odd = torch.zeros(c.n, 256 + 4, dtype=BF16, device=DEV)[:, :256]  # rows not 16-byte aligned
    with pytest.raises(vb.VerillmError) as e:
        vb.op_attention_paged(odd, cache, rows)
    assert e.value.code == vb.E_SHAPE
    long = vb.PagedRows(rows.page_table[:, :1].repeat(1, 60), rows.cu_rows, rows.kv_len, 2)  # 960 positions may be split
    for ws in (torch.empty(64, dtype=torch.uint8, device=DEV), torch.empty(1 << 28, dtype=torch.uint8, device=DEV)[16:]):
        with pytest.raises(vb.VerillmError) as e:
            vb.op_attention_paged(c.dq, cache, long, workspace=ws)
        assert e.value.code == vb.E_SHAPE
    with pytest.raises(vb.VerillmError) as e:
        vb.op_attention_paged(c.dq[:, :192], cache, rows)  # 3 query heads over 2 kv heads
    assert e.value.code == vb.E_SHAPE
    rows.check()


def test_descriptions_are_fixed_and_head_shapes_checked():
    c = Case(E4M3, 4, 2, 64, 16, [2], [20], seed=25, strided=False)
    cache, rows = c.device()
    for obj, name in ((rows, "kv_len"), (rows, "max_rows"), (rows, "page_table"), (cache, "k"), (cache, "v_scale")):
        with pytest.raises(AttributeError):
            setattr(obj, name, getattr(obj, name))
    q3 = c.dq.reshape(c.n, 4, 64)
    assert torch.equal(vb.op_attention_paged(q3, cache, rows)[:2], vb.op_attention_paged(c.dq, cache, rows)[:2])
    for bad in (c.dq.reshape(c.n, 2, 128), c.dq.reshape(c.n, 4, 2, 32), c.dq.flatten(), c.dq[:, :200], c.dq[:, :0]):
        with pytest.raises((ValueError, vb.VerillmError)):
            vb.op_attention_paged(bad, cache, rows)
    with pytest.raises(ValueError):
        vb.kv_write(cache, rows, c.dk_new.reshape(c.n, 1, 128), c.dv_new.reshape(c.n, 1, 128))
    q = c.dq.contiguous()
    with pytest.raises(vb.VerillmError) as e:
        vb.op_attention_paged(q, cache, rows, out=q)
    assert e.value.code == vb.E_INVAL


@pytest.mark.parametrize("dtype", DTYPES)
def test_pools_of_more_than_four_gigabytes(dtype):
    """Pages at the far end of pools whose byte offsets pass 32 bits: writing, reading, and both attention kernels."""
    for rows, kv in (([1, 3], [200, 90]), ([40, 70], [200, 90])):
        c = Case(dtype, 8, 8, 128, 256, rows, kv, seed=26)
        n = c.k.shape[0]
        small, r = c.device()
        pages = (5 << 30) // (8 * 256 * 128 * small.k.element_size())
        big = [torch.empty((pages,) + tuple(t.shape[1:]), dtype=t.dtype, device=DEV) for t in (small.k, small.v)]
        scales = [None if t is None else torch.empty((pages,) + tuple(t.shape[1:]), device=DEV) for t in (small.k_scale, small.v_scale)]
        for dst, src in zip(big + scales, (small.k, small.v, small.k_scale, small.v_scale)):
            if dst is not None:
                dst[pages - n:] = src
        cache = vb.KVCache(*big, *scales)
        far = vb.PagedRows(torch.where(r.page_table < n, r.page_table + (pages - n), r.page_table), r.cu_rows, r.kv_len, r.max_rows, r.status)
        used = int(c.cu[-1])
        assert torch.equal(vb.op_attention_paged(c.dq, cache, far)[:used], vb.op_attention_paged(c.dq, small, r)[:used])
        vb.kv_write(cache, far, c.dk_new, c.dv_new)
        vb.kv_write(small, r, c.dk_new, c.dv_new)
        for got, want in zip(vb.kv_read(cache, far, used), vb.kv_read(small, r, used)):
            assert torch.equal(got, want)
        far.check()
        del cache, big, scales


def test_two_calls_at_once_and_replayed_chunks():
    """A chunk and a decode step side by side on two streams, each with its own workspace, eagerly and as captured graphs
    replayed after the cache, the lengths and the queries changed: the bits of the calls made one after the other."""
    for dtype in DTYPES:
        a = Case(dtype, 32, 8, 128, 16, [200, 60], [900, 700], seed=27, pad=0)
        b = Case(dtype, 32, 8, 128, 16, [1] * 20, [1000 + 50 * i for i in range(20)], seed=28, pad=0)
        calls = []
        for c in (a, b):
            cache, rows = c.device()
            ws = torch.empty(vb.attention_paged_workspace(cache, rows, c.n, 32), dtype=torch.uint8, device=DEV)
            q, out = c.dq.clone(), torch.zeros(c.n, 32 * 128, dtype=BF16, device=DEV)
            calls.append((cache, rows, ws, q, out, c))
        alone = [vb.op_attention_paged(q, cache, rows) for cache, rows, ws, q, out, c in calls]
        streams = [torch.cuda.Stream() for _ in calls]
        torch.cuda.synchronize()
        for _ in range(20):
            for st, (cache, rows, ws, q, out, c) in zip(streams, calls):
                vb.op_attention_paged(q, cache, rows, out=out, workspace=ws, stream=st)
        torch.cuda.synchronize()
        for want, call in zip(alone, calls):
            assert torch.equal(call[4], want)
        graphs = []
        for cache, rows, ws, q, out, c in calls:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                vb.kv_write(cache, rows, c.dk_new, c.dv_new)
                vb.op_attention_paged(q, cache, rows, out=out, workspace=ws)
            graphs.append(graph)
        for step in range(3):
            want = []
            for cache, rows, ws, q, out, c in calls:
                q.mul_(-1.0 if step else 0.5)
                rows.kv_len.sub_(7)
                c.dk_new.mul_(0.5)
                out.zero_()
                vb.kv_write(cache, rows, c.dk_new, c.dv_new)
                want.append(vb.op_attention_paged(q, cache, rows))
            torch.cuda.synchronize()
            for st, graph in zip(streams, graphs):
                with torch.cuda.stream(st):
                    graph.replay()
                    graph.replay()
            torch.cuda.synchronize()
            for call, w in zip(calls, want):
                call[1].check()
                assert torch.equal(call[4], w)


# --------------------------------------------------------------------------- edge cases inside large calls


class LargeCase(Case):
    """The sequences of a test followed by so many others that the kernel for many rows takes the call."""

    def __init__(self, dtype, rows, kv, seed, dh=128):
        super().__init__(dtype, 8, 2, dh, 16, list(rows) + [20] * 150, list(kv) + [40] * 150, seed=seed)

    def device(self):
        cache, rows = super().device()
        sms = torch.cuda.get_device_properties(0).multi_processor_count
        assert vb.attention_paged_workspace(cache, rows, self.n, 8) >= 2 * sms * 256 * (self.dh + 2) * 4
        return cache, rows

    def verify(self):
        cache, rows = self.device()
        lse = torch.zeros(self.n, self.H, device=DEV)
        got = vb.op_attention_paged(self.dq, cache, rows, lse=lse)
        rows.check()
        ref, tol, lref, ltol = self.attention()
        used = int(self.cu[-1])
        assert_within(got[:used].reshape(used, self.H, self.dh), ref[:used], tol[:used], "out")
        assert_within(lse[:used], lref[:used], ltol[:used], "lse")
        return ref[:used]


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
def test_large_call_lengths(dtype, dh):
    LargeCase(dtype, [20, 3, 0, 1, 40, 65, 64, 7], [12, 0, 20, 1, 40, 129, 300, 7], seed=30, dh=dh).verify()


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_call_non_finite_entries(dtype):
    c = LargeCase(dtype, [6, 40], [100, 40], seed=31)
    k, v = (t.float() if dtype == BF16 else t.float() * s[..., None] for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    place = lambda b, p: (int(c.table[b, p // c.ps]), p % c.ps)  # noqa: E731
    (pg, off), (pg1, off1), (pg2, off2) = place(0, 99), place(1, 38), place(1, 39)
    v[pg, 0, off, 5] = float("nan")
    v[pg1, 1, off1, 100] = float("inf")
    k[pg2, 0, off2, 0] = float("nan")
    c.set_pools(k.to(BF16), v.to(BF16))
    ref = c.verify()
    assert not bool(ref.isfinite().all()) and bool(ref.isfinite().any())


@pytest.mark.parametrize("q_size,k_size", [(0.0, 1e-6), (0.0, 0.0), (1e-30, 1e-3), (1e25, 1e-25)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_large_call_very_small_and_large_queries_and_keys(dtype, q_size, k_size):
    c = LargeCase(dtype, [6, 40], [300, 140], seed=32)
    k, v = (t.float() if dtype == BF16 else t.float() * s[..., None] for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    c.set_pools((k.nan_to_num(0.0) * k_size).to(BF16), v.to(BF16))
    c.q.copy_(c.q.float() * q_size)
    c.verify()


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_call_large_scores_and_a_late_maximum(dtype):
    c = LargeCase(dtype, [2, 20], [700, 400], seed=33)
    k, v = (t.float() if dtype == BF16 else t.float() * s[..., None] for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    for b in range(2):
        for p in range(c.kv[b]):
            k[int(c.table[b, p // 16]), :, p % 16] *= 0.02 * p
    c.set_pools(k.to(BF16), v.to(BF16))
    c.verify()


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_call_problems_only_the_device_sees(dtype):
    c = LargeCase(dtype, [50, 50], [64, 64], seed=34)
    cache, r = c.device()
    out = torch.zeros(c.n, 8 * 128, dtype=BF16, device=DEV)
    ref, tol, _, _ = c.attention()
    good = r.page_table.clone()
    for bad in (cache.n_pages, -1, 1 << 30):
        r.page_table[1, 3] = bad
        r.status.zero_()
        vb.op_attention_paged(c.dq, cache, r, out=out)
        assert int(r.status.item()) == vb.DEV_PAGE_RANGE
        assert_within(out[:50].reshape(50, 8, 128), ref[:50], tol[:50])
        assert_within(out[100:c.n - 3].reshape(-1, 8, 128), ref[100:c.n - 3], tol[100:c.n - 3])
    r.page_table.copy_(good)
    r.page_table.clamp_(0, cache.n_pages - 1)
    for length in (-3, 1 << 30):
        r.kv_len[1] = length
        r.status.zero_()
        vb.op_attention_paged(c.dq, cache, r, out=out)
        assert int(r.status.item()) == vb.DEV_ROWS_RANGE
        assert_within(out[:50].reshape(50, 8, 128), ref[:50], tol[:50])


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_block_of_many_rows_over_a_long_context(dtype):
    """A single block whose tiles lie in most CTAs, and one beside a short sequence: the spread join of large blocks."""
    for rows, kv in (([16], [16000]), ([30, 1, 7], [9001, 3, 500])):
        c = Case(dtype, 8, 1, 128, 64, rows, kv, seed=35)
        cache, r = c.device()
        got = vb.op_attention_paged(c.dq, cache, r)
        r.check()
        ref, tol, _, _ = c.attention()
        used = int(c.cu[-1])
        assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used])


@pytest.mark.parametrize("dtype", DTYPES)
def test_non_finite_entries_of_joined_contexts(dtype):
    """Contexts whose pieces are joined, by few CTAs and by many: a NaN key early on, an infinite value among the last."""
    c = Case(dtype, 8, 2, 128, 16, [1, 3, 2], [3000, 9000, 700], seed=36)
    k, v = (t.float() if dtype == BF16 else t.float() * s[..., None] for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)))
    for t, b, p, head, value in ((k, 0, 130, 0, float("nan")), (v, 0, 2000, 1, float("inf")), (v, 1, 8998, 0, -float("inf")), (k, 2, 699, 1, float("nan"))):
        t[int(c.table[b, p // c.ps]), head, p % c.ps, 7] = value
    c.set_pools(k.to(BF16), v.to(BF16))
    cache, rows = c.device()
    got = vb.op_attention_paged(c.dq, cache, rows)
    rows.check()
    ref, tol, _, _ = c.attention()
    used = int(c.cu[-1])
    assert not bool(ref[:used].isfinite().all()) and bool(ref[:used].isfinite().any())
    assert_within(got[:used].reshape(used, c.H, c.dh), ref[:used], tol[:used])
