// Paged key/value cache: what its kernels share.  Sequence description with its device-side checks, the walk
// over the attention work of a batch, and the layout of the partial results of split work.
//
// Work of a batch: rows are packed per kv head ((token, query head of the group), token-major); a block is `tb`
// tokens (a power of two) of one (sequence, kv head), and walks the key tiles of kTile positions up to the last
// position one of its rows may see.  All tiles of all blocks form one line, ordered (sequence, kv head, block,
// tile); CTA c takes tiles [c per, (c + 1) per) of that line, whatever the lengths are, which balances a batch of
// very different lengths and splits a single long sequence over the whole GPU.  A block whose tiles lie in
// several CTAs leaves fp32 partial results (maximum, sum, unnormalised output), at most one block that began
// in an earlier CTA ("head" slot) and one that continues in the next ("tail" slot) per CTA; a second kernel joins
// them in an order that the sizes fix, so that results do not depend on timing.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "kernels.h"

namespace vl {

// One sequence as the device sees it: its packed rows [row0, row0 + n) and its cached positions.
struct SeqView {
    int row0, n, len;
};

__device__ __forceinline__ void raise_status(int* status, int code) {
    if (status) atomicCAS(status, 0, code);
}

// Reads a sequence's description and bounds it to what the buffers hold; anything out of bounds is reported.
__device__ __forceinline__ SeqView load_seq(const PagedRowsDev& r, int page_shift, int b, int* status) {
    const int c0 = __ldg(r.cu_rows + b), c1 = __ldg(r.cu_rows + b + 1), len = __ldg(r.kv_len + b);
    SeqView s;
    s.row0 = min(max(c0, 0), r.n_rows);
    s.n = min(max(c1, s.row0), r.n_rows) - s.row0;
    const long long cap = static_cast<long long>(r.table_width) << page_shift;
    s.len = len < 0 ? 0 : static_cast<int>(min(static_cast<long long>(len), cap));
    if (c0 < 0 || c1 < c0 || c1 > r.n_rows || s.n > r.max_rows || s.len != len) raise_status(status, VERILLM_DEV_ROWS_RANGE);
    if (s.n > r.max_rows) s.n = 0;
    return s;
}

// Page of the sequence's position `pos`; a page outside the pool is reported and read as page 0.
__device__ __forceinline__ int load_page(const PagedRowsDev& r, int page_shift, int n_pages, int b, int pos, int* status) {
    const int page = __ldg(r.page_table + static_cast<size_t>(b) * r.table_width + (pos >> page_shift));
    if (static_cast<unsigned>(page) < static_cast<unsigned>(n_pages)) return page;
    raise_status(status, VERILLM_DEV_PAGE_RANGE);
    return 0;
}

// sum_{y=1..z} ceil(y / 2^s)
__host__ __device__ __forceinline__ long long sum_ceil(long long z, int s) {
    const long long m = z >> s;
    return ((m * (m + 1)) >> 1) * (1LL << s) + (z - (m << s)) * (m + 1);
}

// A kernel's tiles hold T = 2^tl key positions.  (With tl = 30 every block is one tile: shares of whole blocks.)
//
// Tiles of the first m blocks of one (sequence, kv head), none of them its last: block i (from 1) ends at position
// ctx + tb i and takes max(1, ceil((ctx + tb i) / T)) tiles.  With tb <= T, ceil((ctx + tb i) / T) =
// ceil(z_i / p), p = T / tb, z_i = ceil(ctx / tb) + i: a sum over consecutive integers; with tb a multiple of T
// the terms are an arithmetic series.
__host__ __device__ __forceinline__ long long tiles_before(int tl, int ctx, int tb_log, long long m) {
    if (m <= 0) return 0;
    if (tb_log <= tl) {
        const long long z0 = (static_cast<long long>(ctx) + (1 << tb_log) - 1) >> tb_log;  // ceil(ctx / tb)
        if (z0 + m <= 0) return m;
        const long long lo = z0 + 1 > 1 ? z0 + 1 : 1;  // first positive z
        return (lo - (z0 + 1)) + sum_ceil(z0 + m, tl - tb_log) - sum_ceil(lo - 1, tl - tb_log);
    }
    const int q = 1 << (tb_log - tl);
    const long long c0 = (static_cast<long long>(ctx) + (1 << tl) - 1) >> tl;
    long long ones = c0 >= 1 ? 0 : (-c0) / q;  // i <= ones: c0 + q i <= 0, one tile each
    if (ones > m) ones = m;
    const long long k = m - ones;
    return ones + k * c0 + q * ((m * (m + 1) - ones * (ones + 1)) >> 1);
}

__host__ __device__ __forceinline__ int block_count(int n, int tb_log) { return (n + (1 << tb_log) - 1) >> tb_log; }
// Tiles of the block that ends before position `end`
__host__ __device__ __forceinline__ int tiles_of_end(int tl, int end) {
    return end > (1 << tl) ? ((end - 1) >> tl) + 1 : 1;
}
// End position (exclusive) of block j
__host__ __device__ __forceinline__ int block_end(const SeqView& s, int tb_log, int j) {
    const int toks = ((j + 1) << tb_log) < s.n ? (j + 1) << tb_log : s.n;
    return s.len - s.n + toks;
}
// All tiles of one (sequence, kv head)
__host__ __device__ __forceinline__ long long tiles_of_head(int tl, const SeqView& s, int tb_log) {
    if (s.n == 0) return 0;
    return tiles_before(tl, s.len - s.n, tb_log, block_count(s.n, tb_log) - 1) + tiles_of_end(tl, s.len);
}

// a / b of numbers that are not negative and mostly fit 32 bits, where the division is much shorter
__device__ __forceinline__ long long short_div(long long a, long long b) {
    return ((a | b) >> 31) == 0 ? static_cast<long long>(static_cast<unsigned>(a) / static_cast<unsigned>(b)) : a / b;
}

// The CTA's share of the line of tiles.
struct WorkShare {
    long long begin, end, total, per;
    int seq;           // sequence that holds `begin`
    long long offset;  // begin's distance from that sequence's first tile
};

// Finds the CTA's share; to be called by all `nthreads` threads (a multiple of 32, at most 1024) of the block.
// Ends with a barrier.
struct ShareScratch {  // in shared memory
    long long warp_sum[32];
    long long offset;
    int seq;
};
__device__ __forceinline__ void find_share(int tl, const PagedRowsDev& r, int page_shift, int n_kv_heads, int tb_log, int nthreads,
                                           ShareScratch* sc, WorkShare& w, int* status) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nwarps = nthreads >> 5;
    int* st0 = blockIdx.x == 0 ? status : nullptr;  // one CTA reports
    auto tiles = [&](int b) -> long long {
        return b < r.batch ? tiles_of_head(tl, load_seq(r, page_shift, b, st0), tb_log) * n_kv_heads : 0;
    };
    const int live = min(nwarps, (r.batch + 31) >> 5);  // the other warps have nothing to add
    // inclusive scan over the block of one value per thread; returns the block's total
    long long mine = 0, incl = 0;
    auto scan = [&](long long v) -> long long {
        incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += u;
        }
        __syncthreads();  // the previous use of warp_sum is over
        if (lane == 31) sc->warp_sum[warp] = incl;
        __syncthreads();
        long long before = 0, total = 0;
        for (int i = 0; i < live; ++i) {
            const long long s = sc->warp_sum[i];
            before += i < warp ? s : 0;
            total += s;
        }
        incl += before;
        return total;
    };
    const bool one_pass = r.batch <= nthreads;
    long long total = 0;
    if (one_pass) {
        mine = tiles(tid);
        total = scan(mine);
    } else {
        long long v = 0;
        for (int b = tid; b < r.batch; b += nthreads) v += tiles(b);
        total = scan(v);
    }
    w.total = total;
    const long long per = short_div(total + gridDim.x - 1, gridDim.x);
    w.per = per;
    w.begin = min(per * blockIdx.x, total);
    w.end = min(w.begin + per, total);
    if (w.begin < w.end) {
        if (one_pass) {
            if (incl - mine <= w.begin && w.begin < incl) {
                sc->seq = tid;
                sc->offset = w.begin - (incl - mine);
            }
        } else {
            long long base = 0;
            for (int b0 = 0; b0 < r.batch && base <= w.begin; b0 += nthreads) {
                mine = tiles(b0 + tid);
                const long long sum = scan(mine);
                const long long first = base + incl - mine;
                if (first <= w.begin && w.begin < first + mine) {
                    sc->seq = b0 + tid;
                    sc->offset = w.begin - first;
                }
                base += sum;
            }
        }
    }
    __syncthreads();
    w.seq = sc->seq;
    w.offset = sc->offset;
}

// Walk over the blocks of a share.  cur: the block's sequence, kv head, block number, its tiles and the part
// [t0, t1) of them that belongs to this CTA.
struct BlockWalk {
    SeqView s;
    int seq, kvh, j, tiles, t0, t1;
    long long at;  // line position of the block's tile 0
};

// Positions the walk on the first block of a (non-empty) share.
__device__ __forceinline__ void walk_begin(int tl, const PagedRowsDev& r, int page_shift, int tb_log, const WorkShare& w, BlockWalk& k) {
    k.seq = w.seq;
    k.s = load_seq(r, page_shift, k.seq, nullptr);
    const long long per_head = tiles_of_head(tl, k.s, tb_log);
    k.kvh = static_cast<int>(short_div(w.offset, per_head));
    const long long x = w.offset - per_head * k.kvh;
    const int ctx = k.s.len - k.s.n;
    int lo = 0, hi = block_count(k.s.n, tb_log) - 1;  // the last block that begins at or before x
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tiles_before(tl, ctx, tb_log, mid) <= x) lo = mid;
        else hi = mid - 1;
    }
    k.j = lo;
    k.tiles = tiles_of_end(tl, block_end(k.s, tb_log, lo));
    k.at = w.begin - (x - tiles_before(tl, ctx, tb_log, lo));
    k.t0 = static_cast<int>(w.begin - k.at);
    k.t1 = static_cast<int>(min(static_cast<long long>(k.tiles), w.end - k.at));
}

// Moves to the next block; false at the end of the share.
__device__ __forceinline__ bool walk_next(int tl, const PagedRowsDev& r, int page_shift, int n_kv_heads, int tb_log, const WorkShare& w,
                                          BlockWalk& k) {
    k.at += k.tiles;
    if (k.at >= w.end) return false;
    if (++k.j == block_count(k.s.n, tb_log)) {
        k.j = 0;
        if (++k.kvh == n_kv_heads) {
            k.kvh = 0;
            do {  // (a later sequence has tiles, as the share does not end here; the bound is for arrays that change meanwhile)
                if (++k.seq >= r.batch) return false;
                k.s = load_seq(r, page_shift, k.seq, nullptr);
            } while (k.s.n == 0);
        }
    }
    k.tiles = tiles_of_end(tl, block_end(k.s, tb_log, k.j));
    k.t0 = 0;
    k.t1 = static_cast<int>(min(static_cast<long long>(k.tiles), w.end - k.at));
    return true;
}

// Partial results.  hdr[2 c]: {pieces, sequence, kv head, block} of the block whose first tiles CTA c holds and whose
// last it does not (pieces 0: none).  Slot 2 c: the block that began before CTA c; slot 2 c + 1: hdr[2 c]'s block.
// hdr[2 c + 1].x (where the join is spread): the CTA in which slot 2 c's block began, if it has more than kJoinAlone pieces and
// is joined by the CTAs of all of them, else -1.
// A slot holds `rows` maxima (log2 units, -inf: no key yet), `rows` sums, and `rows` x head_dim outputs.
constexpr int kJoinAlone = 16;
__device__ __forceinline__ int last_cta(const WorkShare& w, const BlockWalk& k) { return static_cast<int>(short_div(k.at + k.tiles - 1, w.per)); }
__device__ __forceinline__ void no_headers(int4* hdr) {
    hdr[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
    hdr[2 * blockIdx.x + 1] = make_int4(-1, 0, 0, 0);
}
__device__ __forceinline__ void first_header(int4* hdr, const WorkShare& w, const BlockWalk& k) {  // k: the share's first block
    const int first = static_cast<int>(short_div(k.at, w.per));
    hdr[2 * blockIdx.x + 1] = make_int4(k.t0 != 0 && last_cta(w, k) - first + 1 > kJoinAlone ? first : -1, 0, 0, 0);
}
__device__ __forceinline__ float* part_slot(float* part, int slot, int rows, int dh) {
    return part + static_cast<size_t>(slot) * rows * (dh + 2);
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// weight of a partial result with maximum m in one with maximum mx >= m (both may be -inf: nothing to weigh)
__device__ __forceinline__ float part_weight(float m, float mx) { return m == -INFINITY ? 0.f : exp2_fast(m - mx); }
// A piece's output times its weight.  An infinite one stays infinite where the weight underflowed to 0, as a NaN does: how the keys
// were divided into pieces must not decide what is lost.
__device__ __forceinline__ float weighted(float x, float w) { return w == 0.f && isinf(x) ? x : x * w; }

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Four codes -> fp16 pairs (0, 1) and (2, 3), exactly.  int8: 0x6400 | (code + 128) is the fp16 number 1152 + code.
template <int DTYPE>
__device__ __forceinline__ uint2 widen4_half(uint32_t w) {
    if (DTYPE == VERILLM_KV_E4M3) {
        uint2 h;
        asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}\n" : "=r"(h.x), "=r"(h.y) : "r"(w));
        return h;
    }
    const uint32_t u = w ^ 0x80808080u;
    const __half2 off = __half2half2(__ushort_as_half(static_cast<unsigned short>(0x6480)));  // 1152
    const uint32_t lo = __byte_perm(u, 0x64646464u, 0x4140), hi = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 a = __hsub2(*reinterpret_cast<const __half2*>(&lo), off), b = __hsub2(*reinterpret_cast<const __half2*>(&hi), off);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// Scales of 8-bit pools enter fp16 operands relative to a power of two: 2^-6 of the one at or below the largest scale m of
// a tile, so that the largest lies in [2^6, 2^7) (scales are at least 2^-119).  A reference is kept while scales
// stay at or below kScaleRefMax of it.
constexpr float kScaleRefMax = 128.f;
__device__ __forceinline__ float scale_ref(float m) { return __uint_as_float((max(__float_as_uint(m) >> 23, 7u) - 6u) << 23); }
// Exponent field e such that |q| 2^(127 - e) lies in [1, 2) for the largest entry, whose 15-bit pattern is given.
__device__ __forceinline__ uint32_t row_exponent(uint32_t abs_bits) { return min(max(abs_bits >> 7, 1u), 253u); }
// largest |x| of 8 packed bf16 values as a 15-bit pattern (ordered like the values; >= 0x7F80: not finite)
__device__ __forceinline__ uint32_t abs_max8(const uint4& x) {
    const uint32_t a = __vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), b = __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu);
    const uint32_t m = __vmaxu2(a, b);
    return max(m & 0xFFFFu, m >> 16);
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

}  // namespace vl
