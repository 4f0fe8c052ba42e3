// Causal grouped-query attention of new tokens over a paged cache, few rows per sequence (decode steps, drafted
// tokens): out_r = sum_j p_j v_j scale^v_j, p = softmax_j(q_r . k_j scale^k_j / sqrt(dh)), j up to r's position.
//
// The work is one pass over the sequences' keys and values, bound by HBM: a cached (position, kv head) costs 4 dh
// bytes in bf16, 2 dh + 8 in 8 bits, and meets only the few rows of its group.  So the kernel is built around
// loads, and the products run on the warp-level tensor instructions, whose tiles fit few rows: S^T = K Q^T and
// O^T = V^T P^T, where 16 keys (or 16 head_dim columns) fill the instruction's rows and NT blocks of 8 query rows its
// columns.  (A 128-row tcgen05 tile would idle in 96 - 124 of its rows here and needs operands staged in shared
// memory.)  Keys and values go from global memory straight into the operand registers, 16 bytes a lane: a lane's
// 16 bytes are consecutive head_dim entries, and because both products sum over (or tile) head_dim in any order,
// the order in which the fragments name them is chosen to fit the loads (Q is laid out once to match).  Each of the
// CTA's four warps takes 16 of a tile's 64 keys and keeps its own running maximum, sum and output; they are joined
// once per block.  8-bit codes are widened to fp16 in registers (both code types are exact there) and the products are
// fp16; key scales multiply the scores and value scales the probabilities, both in fp32.  To fit fp16, a query row is
// scaled by a power of two into [1, 2), and value scales are taken relative to a power of two that follows the largest
// seen: a probability times its scale is below 2^15 and loses at most 2^-25, 2^-31 of the largest.
//
// The running maximum is a reference that is only raised when a score exceeds it by 2^8, as in the packed
// attention kernel: probabilities stay below 256 and the sum divides the stale reference out.  Probabilities (times
// scales) are rounded to fp16 for the second product with 8-bit pools; with bf16 pools they enter it as the sum of two
// bf16 numbers (16 significant bits), whose second product hides under the loads (114.4 -> 114.8 us for 64 contexts of
// 2600 on average, and the error of the result falls from 2.3e-3 to the 1.7e-3 of its own rounding).  All else is fp32.
//
// Measured, join included: one row of each of 64 contexts of up to 4096, 32 query heads on 8 of 128, bf16: 116 us = 6.0 TB/s, 92 - 93 %
// of a copy's rate; two contexts of 131072, 64 query heads, e4m3: 100.5 us = 5.3 TB/s; five drafted rows of 16 contexts of up to
// 8192, int8: 70 us = 2.7 TB/s, where 24 rows of output and the keys and values in flight take 255 registers and eight
// warps per SM wait for their own instructions.
#include <algorithm>

#include "paged.cuh"

namespace vl {

namespace {

constexpr int PR_THREADS = 128;
constexpr int PR_WARPS = 4;
constexpr int PR_TILE_LOG = 6, PR_TILE = 1 << PR_TILE_LOG;  // keys per tile: 16 per warp
constexpr float PR_RAISE_LOG2 = 8.f;

// d += a b, 16 x 8 x 16, operands bf16 or fp16
template <bool BF16>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 transpose of 16-bit values over the warp
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// Whether one of 8 packed bf16 values is infinite or NaN, and the 8 values with those replaced by 0.
__device__ __forceinline__ bool not_finite8(const uint4& x) {
    const uint32_t m = __vmaxu2(__vmaxu2(x.x & 0x7F807F80u, x.y & 0x7F807F80u), __vmaxu2(x.z & 0x7F807F80u, x.w & 0x7F807F80u));
    return (m >> 16) == 0x7F80u || (m & 0xFFFFu) == 0x7F80u;
}
__device__ __forceinline__ uint32_t finite2(uint32_t w) {
    if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
    if ((w & 0x7F800000u) == 0x7F800000u) w &= 0x0000FFFFu;
    return w;
}
__device__ __forceinline__ uint4 finite8(const uint4& x) { return make_uint4(finite2(x.x), finite2(x.y), finite2(x.z), finite2(x.w)); }

// How a warp holds 16 keys and 16 values (lane = 4 g + t).
// Keys: lane loads KBYTES of rows g and g + 8 per chunk of 4 KBYTES; 32 bytes where the row has them, so that the four
// lanes of a row take a whole line at a time (8 rows x 64 bytes per load kept the L1 busy twice as long).
// Values: lane loads VB bytes of rows 2t, 2t + 1, 2t + 8, 2t + 9; the 8 lanes g cover VB * 8 bytes of a row.
template <int DH, int DTYPE>
struct Layout {
    static constexpr bool BF16 = DTYPE == VERILLM_KV_BF16;
    static constexpr int ROW_BYTES = DH * (BF16 ? 2 : 1);
    static constexpr int KBYTES = ROW_BYTES >= 128 ? 32 : 16;
    static constexpr int KWORDS = KBYTES / 4;
    static constexpr int KCHUNKS = ROW_BYTES / (4 * KBYTES);
    static constexpr int KSTEPS = DH / 16;
    static constexpr int KSTEP_WORDS = BF16 ? 2 : 1;  // words of a lane and row per step of 16 entries
    // the 4 entries of a row that lane t names in step ks
    static __device__ __forceinline__ int entry(int ks, int t) {
        constexpr int per_chunk = KWORDS / KSTEP_WORDS, lane_entries = KBYTES / (BF16 ? 2 : 1);
        return (ks / per_chunk) * 4 * lane_entries + t * lane_entries + 4 * (ks % per_chunk);
    }
    static constexpr int VPIECES = ROW_BYTES >= 128 ? ROW_BYTES / 128 : 1;  // 16-byte pieces per lane and row
    static constexpr int VWORDS = ROW_BYTES >= 128 ? 4 : 2;                 // words per piece (8-byte pieces: 64 8-bit entries)
    static constexpr int MT = DH / 16;                                      // m tiles of O^T
    // the two head_dim columns a lane holds of m tile i, and i + 1 follows on in the same 16 bytes
    static __device__ __forceinline__ int col(int i, int g) {
        if (!BF16 && DH == 128) return 16 * g + 2 * i;
        return (i >> 2) * 64 + 8 * g + 2 * (i & 3);
    }
};

// a lane's words of a row: 16 or (aligned) 32 bytes
__device__ __forceinline__ void load_words(uint32_t (&w)[4], const char* p) {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(p));
    w[0] = x.x;
    w[1] = x.y;
    w[2] = x.z;
    w[3] = x.w;
}
__device__ __forceinline__ void load_words(uint32_t (&w)[8], const char* p) {
    asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
}

// Adds the infinite and NaN values among a warp's keys to the outputs [row][head_dim] (in shared memory, stride ld) of the rows that
// may see them.
template <int DH>
__device__ __forceinline__ void add_stray(const PagedAttnParams& p, const BlockWalk& k, int warp, int lane, int rows, int first_pos, int end, float* out, int ld) {
    const int shift = p.c.page_shift;
    __syncwarp();  // the lanes wrote other columns than the ones they look at here
#pragma unroll 1
    for (int tile = k.t0; tile < k.t1; ++tile) {
        const int key0 = tile * PR_TILE + warp * 16;
        if (key0 >= end) break;
        const int page = load_page(p.r, shift, p.c.n_pages, k.seq, key0, nullptr);
        const size_t vec = ((static_cast<size_t>(page) * p.c.n_kv_heads + k.kvh) << shift) + (key0 & ((1 << shift) - 1));
#pragma unroll 1
        for (int i = 0; i < 16 && key0 + i < end; ++i) {
            const unsigned short* v = reinterpret_cast<const unsigned short*>(p.c.v) + (vec + i) * DH;
#pragma unroll 1
            for (int col = lane; col < DH; col += 32) {
                const float x = bf16_bits_to_float(__ldg(v + col));
                if (isfinite(x)) continue;
#pragma unroll 1
                for (int r = 0; r < rows; ++r)
                    if (key0 + i <= first_pos + r / p.group) out[r * ld + col] += x;
            }
        }
    }
}

// CTAs per SM, all resident at once: what the registers allow (65536 / 128 threads / CTAs).
__host__ __device__ constexpr int rows_ctas(int dh, int dtype, int nt) {
    if (dh == 64) return nt <= 2 ? 4 : 2;
    return dtype == VERILLM_KV_BF16 ? (nt == 1 ? 3 : 2) : (nt == 1 ? 4 : nt == 2 ? 3 : 2);
}

template <int DH, int DTYPE, int NT>
__global__ void __launch_bounds__(PR_THREADS, rows_ctas(DH, DTYPE, NT))
paged_rows_kernel(const PagedAttnParams p) {
    using L = Layout<DH, DTYPE>;
    constexpr int RB = 8 * NT;
    constexpr int OLD = DH + 4;  // row stride of the joined outputs in shared memory
    extern __shared__ __align__(16) float pr_smem[];
    float* sm_m = pr_smem;                              // [PR_WARPS][RB]
    float* sm_l = sm_m + PR_WARPS * RB;                 // [PR_WARPS][RB]
    float* sm_o = sm_l + PR_WARPS * RB;                 // [PR_WARPS][RB][OLD]
    uint2* sm_q = reinterpret_cast<uint2*>(sm_o + PR_WARPS * RB * OLD);  // [NT][KSTEPS][32]
    __shared__ ShareScratch sm_share;
    __shared__ uint32_t sm_exp[RB];  // 8-bit pools: the query rows' exponents

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const PagedCacheDev& c = p.c;
    const int G = p.group, shift = c.page_shift, ps_mask = (1 << shift) - 1;

    WorkShare share;
    find_share(p.share_log, p.r, shift, c.n_kv_heads, p.tb_log, PR_THREADS, &sm_share, share, p.status);
    pdl_launch_dependents();
    if (share.begin >= share.end) {
        if (tid == 0 && p.hdr) no_headers(p.hdr);
        return;
    }
    BlockWalk k;
    walk_begin(p.share_log, p.r, shift, p.tb_log, share, k);
    const float sl2 = rsqrtf(static_cast<float>(DH)) * kLog2e;
    int4 header = make_int4(0, 0, 0, 0);
    if (tid == 0 && p.hdr) first_header(p.hdr, share, k);

    do {
        const SeqView s = k.s;
        const int tok0 = k.j << p.tb_log, toks = min(1 << p.tb_log, s.n - tok0);
        const int rows = toks * G;  // <= RB
        const int ctx = s.len - s.n;
        const int first_pos = ctx + tok0;         // position of the block's first token
        const int end = ctx + tok0 + toks;        // keys [0, end) are visible to some row
        if (!p.hdr) k.t1 = tiles_of_end(PR_TILE_LOG, end);  // a share of whole blocks: in tiles of this kernel's size
        // ---- Q into fragment order: b registers of k step ks, rows 8 nt + g
        __syncthreads();  // the previous block's rows have been read
        const __nv_bfloat16* q0 = reinterpret_cast<const __nv_bfloat16*>(p.q) + static_cast<size_t>(s.row0 + tok0) * p.q_stride + static_cast<size_t>(k.kvh * G) * DH;
        if (!L::BF16) {
            constexpr int LPQ = NT == 1 ? 16 : NT == 2 ? 8 : 4;  // lanes per row
            const int r = tid / LPQ;
            uint32_t mx = 0;
            if (r < rows) {
                const uint4* src = reinterpret_cast<const uint4*>(q0 + static_cast<size_t>(r / G) * p.q_stride + static_cast<size_t>(r % G) * DH);
                for (int i = tid % LPQ; i < DH / 8; i += LPQ) mx = max(mx, abs_max8(__ldg(src + i)));
            }
#pragma unroll
            for (int x = 1; x < LPQ; x <<= 1) mx = max(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, x));
            if (r < RB && tid % LPQ == 0) sm_exp[r] = row_exponent(mx);
            __syncthreads();
        }
        for (int i = tid; i < NT * L::KSTEPS * 32; i += PR_THREADS) {
            const int ln = i & 31, ks = (i >> 5) % L::KSTEPS, nt = i / (32 * L::KSTEPS);
            const int r = 8 * nt + (ln >> 2), lt = ln & 3;
            uint2 b = make_uint2(0u, 0u);
            if (r < rows) {
                const __nv_bfloat16* src = q0 + static_cast<size_t>(r / G) * p.q_stride + static_cast<size_t>(r % G) * DH;
                const uint2 x = __ldg(reinterpret_cast<const uint2*>(src + L::entry(ks, lt)));
                if (L::BF16) {
                    b = x;
                } else {
                    const float down = __uint_as_float((254u - sm_exp[r]) << 23);
                    b = make_uint2(pack_half(bf16_lo(x.x) * down, bf16_hi(x.x) * down), pack_half(bf16_lo(x.y) * down, bf16_hi(x.y) * down));
                }
            }
            sm_q[i] = b;
        }
        __syncthreads();

        float o[NT][L::MT][4], m_ref[NT][2], l_run[NT][2], rf[NT][2], vref = 0.f, vup = 0.f;
        int pos[NT][2];  // last visible key of this lane's rows, -1: none
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < L::MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 8 * nt + 2 * t + h;
                pos[nt][h] = r < rows ? first_pos + r / G : -1;
                rf[nt][h] = L::BF16 ? sl2 : sl2 * __uint_as_float(r < rows ? sm_exp[r] << 23 : 0u);
                m_ref[nt][h] = -INFINITY;
                l_run[nt][h] = 0.f;
            }
        }

        uint32_t ka[L::KCHUNKS][L::KWORDS], kb[L::KCHUNKS][L::KWORDS];
        uint4 v[L::VPIECES][4];
        float ks0 = 1.f, ks1 = 1.f, vs0 = 1.f, vs1 = 1.f, vs0n = 1.f, vs1n = 1.f;
        auto token_of = [&](int tile) { return tile * PR_TILE + warp * 16; };
        auto load_keys = [&](size_t vec) {
            const char* base = reinterpret_cast<const char*>(c.k) + (vec + g) * L::ROW_BYTES + t * L::KBYTES;
#pragma unroll
            for (int i = 0; i < L::KCHUNKS; ++i) {
                load_words(ka[i], base + i * 4 * L::KBYTES);
                load_words(kb[i], base + 8 * L::ROW_BYTES + i * 4 * L::KBYTES);
            }
            if (!L::BF16) {
                ks0 = __ldg(c.k_scale + vec + g);
                ks1 = __ldg(c.k_scale + vec + 8 + g);
                vs0n = __ldg(c.v_scale + vec + g);
                vs1n = __ldg(c.v_scale + vec + 8 + g);
            }
        };
        auto load_values = [&](size_t vec) {
            const char* base = reinterpret_cast<const char*>(c.v) + (vec + 2 * t) * L::ROW_BYTES + g * (4 * L::VWORDS);
#pragma unroll
            for (int i = 0; i < L::VPIECES; ++i) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const char* src = base + ((e & 1) + 8 * (e >> 1)) * L::ROW_BYTES + i * 128;
                    if (L::VWORDS == 4) {
                        v[i][e] = __ldg(reinterpret_cast<const uint4*>(src));
                    } else {
                        const uint2 x = __ldg(reinterpret_cast<const uint2*>(src));
                        v[i][e] = make_uint4(x.x, x.y, 0u, 0u);
                    }
                }
            }
        };

        // Page numbers are read ahead.  With 8-bit pools, whose tiles bring half the bytes, they are read three tiles ahead
        // and the tile two ahead is asked into L2 (a line per lane), so that the register loads, one tile ahead, find a
        // short way: 112 -> 100 us for two contexts of 131072.  bf16 has enough in flight without, and reads them one tile
        // ahead (64 contexts of 2600 on average: 114 us, 119 with the longer chain).
        auto page_at = [&](int key) { return key < min(end, k.t1 << PR_TILE_LOG) ? load_page(p.r, shift, c.n_pages, k.seq, key, p.status) : 0; };
        auto vec_in = [&](int page, int key) -> size_t { return ((static_cast<size_t>(page) * c.n_kv_heads + k.kvh) << shift) + (key & ps_mask); };
        auto prefetch = [&](size_t vec) {
            const char* row = reinterpret_cast<const char*>(lane < 16 ? c.k : c.v) + (vec + (lane & 15)) * L::ROW_BYTES;
#pragma unroll
            for (int i = 0; i < L::ROW_BYTES; i += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + i));
        };
        int tile = k.t0;
        bool stray = false;  // bf16 pools: some value of this warp's was not finite
        size_t vec_next = 0;
        int page2 = 0;
        {
            const int key = token_of(tile);
            const int page0 = page_at(key), page1 = L::BF16 ? 0 : page_at(key + PR_TILE);
            if (!L::BF16) page2 = page_at(key + 2 * PR_TILE);
            const size_t vec = vec_in(page0, key);
            vec_next = vec_in(page1, key + PR_TILE);
            if (key < end) {
                load_keys(vec);
                load_values(vec);
            }
            if (!L::BF16 && tile + 1 < k.t1 && key + PR_TILE < end) prefetch(vec_next);
        }
        for (; tile < k.t1; ++tile) {
            const int key0 = token_of(tile);
            if (key0 >= end) break;  // the same for every later tile
            const bool more = tile + 1 < k.t1 && key0 + PR_TILE < end;
            size_t vec2 = 0;
            if (L::BF16) {
                vec_next = vec_in(page_at(key0 + PR_TILE), key0 + PR_TILE);
            } else {
                vec2 = vec_in(page2, key0 + 2 * PR_TILE);
                if (tile + 2 < k.t1 && key0 + 2 * PR_TILE < end) prefetch(vec2);
                page2 = page_at(key0 + 3 * PR_TILE);
            }
            // ---- S^T = K Q^T: 16 keys x 8 NT rows
            float sc[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < L::KSTEPS; ++ks) {
                constexpr int per_chunk = L::KWORDS / L::KSTEP_WORDS;
                const int i = ks / per_chunk, w = (ks % per_chunk) * L::KSTEP_WORDS;
                uint2 a, e;  // rows g and g + 8
                if (L::BF16) {
                    a = make_uint2(ka[i][w], ka[i][(w + 1) % L::KWORDS]);
                    e = make_uint2(kb[i][w], kb[i][(w + 1) % L::KWORDS]);
                } else {
                    a = widen4_half<DTYPE>(ka[i][w]);
                    e = widen4_half<DTYPE>(kb[i][w]);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint2 b = sm_q[(nt * L::KSTEPS + ks) * 32 + lane];
                    mma16<L::BF16>(sc[nt], a.x, e.x, a.y, e.y, b.x, b.y);
                }
            }
            const float f0 = ks0, f1 = ks1;
            vs0 = vs0n;
            vs1 = vs1n;
            if (more) load_keys(vec_next);
            // ---- mask, running maximum, probabilities
            const bool masked = key0 + 15 > first_pos;  // some row may not see some key of the 16
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    sc[nt][h] *= L::BF16 ? sl2 : f0 * rf[nt][h];
                    sc[nt][2 + h] *= L::BF16 ? sl2 : f1 * rf[nt][h];
                }
                if (masked) {  // (rows past the block's last hold zeros and are not written)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (key0 + g > pos[nt][h]) sc[nt][h] = -INFINITY;
                        if (key0 + 8 + g > pos[nt][h]) sc[nt][2 + h] = -INFINITY;
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) raise |= fmaxf(sc[nt][h], sc[nt][2 + h]) > m_ref[nt][h] + PR_RAISE_LOG2;
            }
            if (!L::BF16) {
                if (key0 + 16 > end) {  // scales behind the last key are whatever the page holds
                    if (key0 + g >= end) vs0 = 0.f;
                    if (key0 + 8 + g >= end) vs1 = 0.f;
                }
                raise |= vref == 0.f || fmaxf(vs0, vs1) > vref * kScaleRefMax;
            }
            if (__any_sync(0xFFFFFFFFu, raise)) {
                float ratio = 1.f;
                if (!L::BF16) {
                    const float ref = fmaxf(vref, scale_ref(warp_max(fmaxf(isfinite(vs0) ? vs0 : 0.f, isfinite(vs1) ? vs1 : 0.f))));
                    ratio = vref / ref;  // at most 1: the reference falls below the largest scale only by its power of two
                    vref = ref;
                    vup = 1.f / ref;  // a power of two, at most 2^126
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float f[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float mx = fmaxf(sc[nt][h], sc[nt][2 + h]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, x));
                        f[h] = 1.f;
                        if (mx > m_ref[nt][h] + PR_RAISE_LOG2) {
                            f[h] = exp2_fast(m_ref[nt][h] - mx);  // 0 for the first keys
                            m_ref[nt][h] = mx;
                        }
                        l_run[nt][h] *= f[h];
                        f[h] *= ratio;
                    }
#pragma unroll
                    for (int i = 0; i < L::MT; ++i) {
                        o[nt][i][0] *= f[0];
                        o[nt][i][1] *= f[1];
                        o[nt][i][2] *= f[0];
                        o[nt][i][3] *= f[1];
                    }
                }
            }
            // values behind the last visible key are whatever the page holds: make them 0
            if (key0 + 16 > end) {
#pragma unroll
                for (int i = 0; i < L::VPIECES; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (key0 + 2 * t + (e & 1) + 8 * (e >> 1) >= end) v[i][e] = make_uint4(0u, 0u, 0u, 0u);
            }
            // An infinite or NaN value must not reach the rows that may not see its token (their probability 0 times it
            // would be NaN), nor meet the remainder of a probability, which may be 0 or negative, nor a probability or factor
            // that underflowed: such entries are taken out of the product here and put into the results at the end, row by row.
            // 8-bit pools carry a non-finite vector in its scale, which is masked with the probability and stays NaN
            // in every product.  (Looking costs 114.4 -> 115.2 us for 64 contexts of up to 4096.)
            if (L::BF16) {
                bool bad = false;
#pragma unroll
                for (int i = 0; i < L::VPIECES; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) bad |= not_finite8(v[i][e]);
                if (__any_sync(0xFFFFFFFFu, bad)) {
                    stray = true;
#pragma unroll
                    for (int i = 0; i < L::VPIECES; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[i][e] = finite8(v[i][e]);
                }
            }
            uint32_t pb[NT][2], pl[NT][2];  // probabilities for the product; bf16: their roundings' remainders too
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float e[4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float ref = m_ref[nt][h] == -INFINITY ? 0.f : m_ref[nt][h];
                    e[h] = exp2_fast(sc[nt][h] - ref);
                    e[2 + h] = exp2_fast(sc[nt][2 + h] - ref);
                    l_run[nt][h] += e[h] + e[2 + h];
                }
                if (!L::BF16) {
                    const float w0 = vs0 * vup, w1 = vs1 * vup;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {  // a masked key's scale may be NaN: 0 stays 0
                        e[h] = masked && key0 + g > pos[nt][h] ? 0.f : e[h] * w0;
                        e[2 + h] = masked && key0 + 8 + g > pos[nt][h] ? 0.f : e[2 + h] * w1;
                    }
                }
                const uint32_t p0 = L::BF16 ? pack_bf16(e[0], e[1]) : pack_half(e[0], e[1]), p1 = L::BF16 ? pack_bf16(e[2], e[3]) : pack_half(e[2], e[3]);
                pb[nt][0] = transpose8(p0);
                pb[nt][1] = transpose8(p1);
                if (L::BF16) {
                    pl[nt][0] = transpose8(pack_bf16(e[0] - bf16_lo(p0), e[1] - bf16_hi(p0)));
                    pl[nt][1] = transpose8(pack_bf16(e[2] - bf16_lo(p1), e[3] - bf16_hi(p1)));
                }
            }
            // ---- O^T += V^T P^T
#pragma unroll
            for (int i = 0; i < L::VPIECES; ++i) {
                const uint32_t w0[4] = {v[i][0].x, v[i][0].y, v[i][0].z, v[i][0].w}, w1[4] = {v[i][1].x, v[i][1].y, v[i][1].z, v[i][1].w};
                const uint32_t w2[4] = {v[i][2].x, v[i][2].y, v[i][2].z, v[i][2].w}, w3[4] = {v[i][3].x, v[i][3].y, v[i][3].z, v[i][3].w};
#pragma unroll
                for (int w = 0; w < L::VWORDS; ++w) {
                    if (L::BF16) {  // a word holds two columns: one m tile
                        const uint32_t a0 = __byte_perm(w0[w], w1[w], 0x5410), a1 = __byte_perm(w0[w], w1[w], 0x7632);
                        const uint32_t a2 = __byte_perm(w2[w], w3[w], 0x5410), a3 = __byte_perm(w2[w], w3[w], 0x7632);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma16<L::BF16>(o[nt][4 * i + w], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
                            mma16<L::BF16>(o[nt][4 * i + w], a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
                        }
                    } else {  // four columns: two m tiles
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            // the two keys of a pair side by side, column by column
                            const uint2 a = widen4_half<DTYPE>(__byte_perm(w0[w], w1[w], h ? 0x7362 : 0x5140));
                            const uint2 e = widen4_half<DTYPE>(__byte_perm(w2[w], w3[w], h ? 0x7362 : 0x5140));
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma16<L::BF16>(o[nt][2 * w + h], a.x, a.y, e.x, e.y, pb[nt][0], pb[nt][1]);
                        }
                    }
                }
            }
            if (more) load_values(vec_next);
            if (!L::BF16) vec_next = vec2;
        }

        // ---- join the four warps: maxima and sums first, then outputs on the common reference
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l_run[nt][h] += __shfl_xor_sync(0xFFFFFFFFu, l_run[nt][h], x);
                if (g == 0) {
                    sm_m[warp * RB + 8 * nt + 2 * t + h] = m_ref[nt][h];
                    sm_l[warp * RB + 8 * nt + 2 * t + h] = l_run[nt][h];
                }
            }
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float f[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 8 * nt + 2 * t + h;
                const float mx = fmaxf(fmaxf(sm_m[r], sm_m[RB + r]), fmaxf(sm_m[2 * RB + r], sm_m[3 * RB + r]));
                f[h] = part_weight(m_ref[nt][h], mx) * (L::BF16 ? 1.f : vref);
            }
#pragma unroll
            for (int i = 0; i < L::MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<float2*>(sm_o + (warp * RB + 8 * nt + 2 * t + h) * OLD + L::col(i, g)) =
                        make_float2(o[nt][i][h] * f[h], o[nt][i][2 + h] * f[h]);
        }
        if (L::BF16 && stray) add_stray<DH>(p, k, warp, lane, rows, first_pos, end, sm_o + warp * RB * OLD, OLD);
        __syncthreads();

        const bool whole = !p.hdr || (k.t0 == 0 && k.t1 == k.tiles);
        const int slot = 2 * blockIdx.x + (k.t0 == 0 ? 1 : 0);
        float* part = whole ? nullptr : part_slot(p.part, slot, RB, DH);
        if (!whole && k.t0 == 0)
            header = make_int4(last_cta(share, k) - static_cast<int>(blockIdx.x) + 1, k.seq, k.kvh, k.j);
        constexpr int LPR = DH / 8;  // lanes per row, 8 columns each
        for (int r = tid / LPR; r < rows; r += PR_THREADS / LPR) {
            const int cx = (tid % LPR) * 8;
            float mx = -INFINITY, l = 0.f;
#pragma unroll
            for (int w = 0; w < PR_WARPS; ++w) mx = fmaxf(mx, sm_m[w * RB + r]);
#pragma unroll
            for (int w = 0; w < PR_WARPS; ++w) l += sm_l[w * RB + r] * part_weight(sm_m[w * RB + r], mx);
            float acc[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = 0.f;
#pragma unroll
            for (int w = 0; w < PR_WARPS; ++w)
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const float4 x = *reinterpret_cast<const float4*>(sm_o + (w * RB + r) * OLD + cx + i);
                    acc[i] += x.x;
                    acc[i + 1] += x.y;
                    acc[i + 2] += x.z;
                    acc[i + 3] += x.w;
                }
            if (whole) {
                const float inv = l == 0.f ? 0.f : 1.f / l;  // no visible key: 0
                const int row = s.row0 + tok0 + r / G, head = k.kvh * G + r % G;
                *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) + static_cast<size_t>(row) * p.out_stride +
                                          static_cast<size_t>(head) * DH + cx) =
                    make_uint4(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv),
                               pack_bf16(acc[4] * inv, acc[5] * inv), pack_bf16(acc[6] * inv, acc[7] * inv));
                if (p.lse && cx == 0) p.lse[static_cast<size_t>(row) * p.n_heads + head] = l == 0.f ? -INFINITY : mx * kLn2 + logf(l);
            } else {
                if (cx == 0) {
                    part[r] = mx;
                    part[RB + r] = l;
                }
                float4* dst = reinterpret_cast<float4*>(part + 2 * RB + r * DH + cx);
                dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
                dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
            }
        }
    } while (walk_next(p.share_log, p.r, shift, c.n_kv_heads, p.tb_log, share, k));
    if (tid == 0 && p.hdr) p.hdr[2 * blockIdx.x] = header;
}

// Joins the partial results of blocks that several CTAs worked on, adding the pieces in the order of their tiles.  The time is
// that of a few dependent reads of L2, so the reads of one step are all in flight together.
//  By the CTAs of the block's first CTA, one for each group of 8 RPW rows, RPW rows per warp: the lanes first look at all
//    pieces' maxima and sums, then each adds its columns of the pieces.  Nothing waits for the sequence's description
//    before the results are stored.
//  Blocks of more than kJoinAlone pieces (few long contexts; SPREAD): by the CTAs of all the CTAs that worked on the block, a
//    row at a time each, the pieces dealt out over the eight warps and these joined last.  One context of 32768, 8 kv heads, bf16:
//    39.1 -> 32.5 us; four of up to 57000, one kv head, int8: 40.1 -> 26.8; two of 131072, 37 pieces: 101.8 -> 100.1.
//    The tcgen05 kernel's 256-row blocks keep many warps busy as it is; their join is spread where there are fewer than
//    grid / kSpreadPieces of them (one block of 128 rows over 16000, 125 pieces: 58 -> 20 us; four over 60000, 37 pieces: 77 -> 67;
//    but with 18 pieces, 64 rows over 32768, 67 would become 77).  The host sees no lengths: a batch of 16 rows of each of eight sequences on
//    one kv head, one over 16000 and seven over 100, has eight blocks and is joined by the long one's few warps, 65 us where 20 would do.
//    Deciding on the device cost the calls that are not spread 59 -> 62 - 65 us (64 rows over 32768) and 592 -> 600 (1024 rows, e4m3).
constexpr int JOIN_THREADS = 256, JOIN_WARPS = JOIN_THREADS / 32;

// The pieces of one block: piece 0 is its first CTA's tail slot, piece i the head slot of the i-th CTA after it.
template <int DH>
struct Pieces {
    static constexpr int W = DH / 32;  // columns per lane
    const float* slot0;
    size_t slot;
    int rows_per_block;
    __device__ __forceinline__ Pieces(const PagedAttnParams& p, int first, int rows)
        : slot0(part_slot(p.part, 2 * first, rows, DH)), slot(static_cast<size_t>(rows) * (DH + 2)), rows_per_block(rows) {}
    __device__ __forceinline__ const float* at(int i) const { return slot0 + slot * (i == 0 ? 1 : 2 * i); }
    __device__ __forceinline__ float maximum(int i, int r) const { return at(i)[r]; }
    __device__ __forceinline__ float sum(int i, int r) const { return at(i)[rows_per_block + r]; }
    __device__ __forceinline__ void columns(int i, int r, int lane, float (&x)[W]) const {
        const float* src = at(i) + 2 * rows_per_block + r * DH + lane * W;
        if (W == 4) {
            const float4 v = *reinterpret_cast<const float4*>(src);
            x[0] = v.x; x[1] = v.y; x[W - 2] = v.z; x[W - 1] = v.w;
        } else {
            const float2 v = *reinterpret_cast<const float2*>(src);
            x[0] = v.x; x[1] = v.y;
        }
    }
};

// Row r of the block that h describes, from its maximum, sum and this lane's columns (by a whole warp).
template <int DH>
__device__ __forceinline__ void put_row(const PagedAttnParams& p, const SeqView& s, const int4& h, int r, int lane, float mx, float l, const float (&acc)[DH / 32]) {
    constexpr int W = DH / 32;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int row = s.row0 + (h.w << p.tb_log) + r / p.group, head = h.z * p.group + r % p.group;
    uint32_t* dst = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(p.out) + static_cast<size_t>(row) * p.out_stride +
                                                static_cast<size_t>(head) * DH + lane * W);
    if (W == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[W - 2] * inv, acc[W - 1] * inv));
    else dst[0] = pack_bf16(acc[0] * inv, acc[1] * inv);
    if (p.lse && lane == 0) p.lse[static_cast<size_t>(row) * p.n_heads + head] = l == 0.f ? -INFINITY : mx * kLn2 + logf(l);
}

// Rows r0 .. r0 + RPW - 1 (of one warp) over the pieces first, first + step, ..: maxima, sums and this lane's columns.
template <int DH, int RPW>
__device__ __forceinline__ void add_pieces(const Pieces<DH>& parts, int n_pieces, int first, int step, int r0, int lane, float (&mx)[RPW], float (&l)[RPW],
                                           float (&acc)[RPW][DH / 32]) {
    constexpr int W = DH / 32;
    constexpr int AHEAD = 8 / RPW;  // pieces in flight
    const int count = (n_pieces - first + step - 1) / step;
    auto piece = [&](int i) { return first + i * step; };
    float m_part[RPW], l_part[RPW];  // of the piece that this lane looks at; read once where there are up to 32
#pragma unroll
    for (int j = 0; j < RPW; ++j) {
        m_part[j] = lane < count ? parts.maximum(piece(lane), r0 + j) : -INFINITY;
        l_part[j] = lane < count ? parts.sum(piece(lane), r0 + j) : 0.f;
        mx[j] = m_part[j];
        l[j] = 0.f;
#pragma unroll
        for (int c = 0; c < W; ++c) acc[j][c] = 0.f;
    }
    for (int i = lane + 32; i < count; i += 32)
#pragma unroll
        for (int j = 0; j < RPW; ++j) mx[j] = fmaxf(mx[j], parts.maximum(piece(i), r0 + j));
#pragma unroll
    for (int j = 0; j < RPW; ++j) mx[j] = warp_max(mx[j]);
    for (int i0 = 0; i0 < count; i0 += 32) {
        const int i = i0 + lane, n = min(32, count - i0);
        float w[RPW];
#pragma unroll
        for (int j = 0; j < RPW; ++j) {
            if (i0 != 0) {
                m_part[j] = i < count ? parts.maximum(piece(i), r0 + j) : -INFINITY;
                l_part[j] = i < count ? parts.sum(piece(i), r0 + j) : 0.f;
            }
            w[j] = part_weight(m_part[j], mx[j]);
            l[j] += warp_sum(l_part[j] * w[j]);
        }
        for (int q0 = 0; q0 < n; q0 += AHEAD) {
            float x[AHEAD][RPW][W];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
#pragma unroll
                for (int j = 0; j < RPW; ++j) parts.columns(piece(i0 + min(q0 + q, n - 1)), r0 + j, lane, x[q][j]);
#pragma unroll
            for (int q = 0; q < AHEAD; ++q)
#pragma unroll
                for (int j = 0; j < RPW; ++j) {
                    const bool one = q0 + q < n;  // uniform; else a repeated read of the last piece
                    const float wq = one ? __shfl_sync(0xFFFFFFFFu, w[j], q0 + q) : 0.f;
#pragma unroll
                    for (int c = 0; c < W; ++c) acc[j][c] += one ? weighted(x[q][j][c], wq) : 0.f;
                }
        }
    }
}

template <int DH>
__device__ __forceinline__ void join_spread(const PagedAttnParams& p, int rows_per_block, const int4& h, int first) {
    constexpr int W = DH / 32;
    __shared__ float sm_m[JOIN_WARPS], sm_l[JOIN_WARPS], sm_o[JOIN_WARPS][DH];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const SeqView s = load_seq(p.r, p.c.page_shift, h.y, nullptr);
    const int rows = min(1 << p.tb_log, s.n - (h.w << p.tb_log)) * p.group;
    const Pieces<DH> parts(p, first, rows_per_block);
    const int units = h.x * gridDim.y, unit = (static_cast<int>(blockIdx.x) - first) * gridDim.y + blockIdx.y;
    for (int r = unit; r < rows; r += units) {
        float mx[1], l[1], acc[1][W];
        add_pieces<DH, 1>(parts, h.x, warp, JOIN_WARPS, r, lane, mx, l, acc);
        if (lane == 0) {
            sm_m[warp] = mx[0];
            sm_l[warp] = l[0];
        }
#pragma unroll
        for (int c = 0; c < W; ++c) sm_o[warp][lane * W + c] = acc[0][c];
        __syncthreads();
        if (warp == 0) {
            float top = -INFINITY, sum = 0.f, o[W] = {};
#pragma unroll
            for (int w = 0; w < JOIN_WARPS; ++w) top = fmaxf(top, sm_m[w]);
#pragma unroll
            for (int w = 0; w < JOIN_WARPS; ++w) {
                const float f = part_weight(sm_m[w], top);
                sum += sm_l[w] * f;
#pragma unroll
                for (int c = 0; c < W; ++c) o[c] += weighted(sm_o[w][lane * W + c], f);
            }
            put_row<DH>(p, s, h, r, lane, top, sum, o);
        }
        __syncthreads();
    }
}

template <int DH, int RPW, bool SPREAD>
__global__ void __launch_bounds__(JOIN_THREADS)
paged_join_kernel(const PagedAttnParams p, int rows_per_block) {
    pdl_wait();
    const int first = static_cast<int>(blockIdx.x);
    const int4 h = p.hdr[2 * first], past = SPREAD ? p.hdr[2 * first + 1] : make_int4(-1, 0, 0, 0);
    if (SPREAD && h.x > kJoinAlone) {
        join_spread<DH>(p, rows_per_block, h, first);
    } else if (h.x > 0) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const int r0 = (static_cast<int>(blockIdx.y) * JOIN_WARPS + warp) * RPW;  // rows_per_block is a multiple of 8 RPW
        const SeqView s = load_seq(p.r, p.c.page_shift, h.y, nullptr);
        float mx[RPW], l[RPW], acc[RPW][DH / 32];
        add_pieces<DH, RPW>(Pieces<DH>(p, first, rows_per_block), h.x, 0, 1, r0, lane, mx, l, acc);
        const int rows = min(1 << p.tb_log, s.n - (h.w << p.tb_log)) * p.group;
#pragma unroll
        for (int j = 0; j < RPW; ++j)
            if (r0 + j < rows) put_row<DH>(p, s, h, r0 + j, lane, mx[j], l[j], acc[j]);  // (what lies behind the block's rows was never written)
    }
    if (SPREAD && past.x >= 0) {
        const int4 begun = p.hdr[2 * past.x];
        if (begun.x > 0) join_spread<DH>(p, rows_per_block, begun, past.x);
    }
}

template <int DH, int NT>
constexpr size_t rows_smem() {
    return static_cast<size_t>(PR_WARPS) * 8 * NT * (2 + DH + 4) * 4 + static_cast<size_t>(NT) * (DH / 16) * 32 * 8;
}

template <int DH, int DTYPE, int NT>
cudaError_t rows_init() {
    return cudaFuncSetAttribute(paged_rows_kernel<DH, DTYPE, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(rows_smem<DH, NT>()));
}
template <int DH, int DTYPE>
cudaError_t rows_init_all() {
    cudaError_t e = rows_init<DH, DTYPE, 1>();
    if (e == cudaSuccess) e = rows_init<DH, DTYPE, 2>();
    if (e == cudaSuccess) e = rows_init<DH, DTYPE, 3>();
    if (e == cudaSuccess && DTYPE != VERILLM_KV_BF16) e = rows_init<DH, DTYPE, (DTYPE != VERILLM_KV_BF16 ? 4 : 3)>();
    return e;
}

template <int DH, int DTYPE, int NT>
cudaError_t rows_launch(const PagedAttnParams& p, int grid, cudaStream_t stream) {
    paged_rows_kernel<DH, DTYPE, NT><<<grid, PR_THREADS, rows_smem<DH, NT>(), stream>>>(p);
    return cudaGetLastError();
}
template <int DH, int DTYPE>
cudaError_t rows_launch_nt(const PagedAttnParams& p, int nt, int grid, cudaStream_t stream) {
    if (nt == 1) return rows_launch<DH, DTYPE, 1>(p, grid, stream);
    if (nt == 2) return rows_launch<DH, DTYPE, 2>(p, grid, stream);
    if (nt == 3) return rows_launch<DH, DTYPE, 3>(p, grid, stream);
    return rows_launch<DH, DTYPE, (DTYPE != VERILLM_KV_BF16 ? 4 : 3)>(p, grid, stream);  // (bf16 takes up to three blocks)
}
template <int DH>
cudaError_t rows_launch_dtype(const PagedAttnParams& p, int nt, int grid, cudaStream_t stream) {
    if (p.c.dtype == VERILLM_KV_BF16) return rows_launch_nt<DH, VERILLM_KV_BF16>(p, nt, grid, stream);
    if (p.c.dtype == VERILLM_KV_E4M3) return rows_launch_nt<DH, VERILLM_KV_E4M3>(p, nt, grid, stream);
    return rows_launch_nt<DH, VERILLM_KV_INT8>(p, nt, grid, stream);
}

// Which kernel and block shape serve a call.  The few-row kernel takes
//  - sequences of up to 24 (bf16) or 32 (8-bit) packed rows, a block each.  Measured for 16 contexts of 4096, 8 kv heads of 128,
//    few-row against tcgen05: bf16 16 rows 61 / 69 us, 24 rows 69 / 70, 32 rows 118 / 70; int8 16 rows 57 / 91, 24 rows
//    61 / 91, 32 rows 80 / 91;
//  - and calls so small that blocks of up to 16 rows give its CTAs one block, or two tiles, each: there the longer pipeline of the
//    tcgen05 kernel counts, not its rate.  64 rows over 250 positions (8 kv heads of 128) bf16 13.0 / 16.0 us, e4m3 13.8 / 18.8; 16
//    rows over 500 e4m3 14.1 / 16.8; 16 rows of 8 heads over 4000 (one kv head) e4m3 19.2 / 25.5.  With five tiles each
//    instead of two: 64 rows over 1000 e4m3 25.5 / 22.6.
// The tcgen05 kernel takes everything else.
struct Shape {
    int nt;  // 8-row column blocks of the few-row kernel; 0: the tcgen05 kernel
    int tb_log, rows_per_block, grid;
    bool split;   // blocks may be split over CTAs and joined
    bool spread;  // tcgen05 kernel: so few blocks that each has many pieces
};
// Contexts of at most kWhole positions (by the table's width: the lengths are on the device) are not split by the few-row kernel:
// four tiles one after the other take as long as a second launch.  Up to kWholeFilled positions, not where the blocks alone keep
// the CTAs busy: at least one for every second SM, and the last round of them three quarters full where they take several.
// Device time, whole / split and joined, us: 32 query heads on 8 of 128, one row over 250 positions: 1 sequence bf16 9.0 / 9.0,
// 16 10.6 / 12.7, 64 e4m3 13.3 / 15.0; over 500: 1 sequence (8 blocks) bf16 12.5 / 9.2, e4m3 13.5 / 10.0; 8 (64 blocks) 12.9 /
// 12.3 and 13.7 / 12.3; 16 (128) 14.1 / 16.4 and 15.0 / 13.9; 32 16.8 / 19.9 and 16.6 / 17.2; 64 (512 blocks on 444 or 592 CTAs) 36.5 /
// 33.4 and 18.4 / 26.6; over 1000: 1 18.8 / 10.6, 16 21.7 / 19.0, 64 60.6 / 54.7.  From a Python loop a split call takes 20 us, a whole
// one 16: a second launch and a workspace.
constexpr long long kWhole = 256, kWholeFilled = 512;
constexpr int kSmallBlockRows = 16;
constexpr long long kSpreadPieces = 32;  // pieces per block from which the tcgen05 kernel's join is spread (see there)
Shape shape_of(const PagedCacheDev& c, const PagedRowsDev& rows, int group, int num_sms) {
    Shape s;
    const long long r = static_cast<long long>(group) * rows.max_rows, positions = static_cast<long long>(rows.table_width) << c.page_shift;
    auto blocks = [&](int tb_log) {  // at most
        const long long per_seq = (rows.max_rows + (1LL << tb_log) - 1) >> tb_log;
        return c.n_kv_heads * std::min(rows.batch * per_seq, (static_cast<long long>(rows.n_rows) >> tb_log) + rows.batch);
    };
    long long whole = kWhole;
    s.tb_log = 0;  // tokens per block: a power of two
    s.nt = 0;
    if (r <= (c.dtype == VERILLM_KV_BF16 ? 24 : 32)) {
        s.nt = static_cast<int>((r + 7) / 8);
        while ((1LL << s.tb_log) < rows.max_rows) ++s.tb_log;  // all of a sequence's
        const long long ctas = static_cast<long long>(num_sms) * rows_ctas(c.head_dim, c.dtype, s.nt), n = blocks(s.tb_log), rounds = (n + ctas - 1) / ctas;
        if (2 * n >= num_sms && (rounds <= 1 || 4 * n >= 3 * rounds * ctas)) whole = kWholeFilled;
    } else if (group <= kSmallBlockRows) {
        int tb_log = 0;
        while ((2 << tb_log) * group <= kSmallBlockRows) ++tb_log;
        const int nt = ((group << tb_log) + 7) / 8;
        const long long ctas = static_cast<long long>(num_sms) * rows_ctas(c.head_dim, c.dtype, nt), n = blocks(tb_log);
        if (positions <= kWhole ? n <= ctas : n * ((positions + PR_TILE - 1) / PR_TILE) <= 2 * ctas) {
            s.nt = nt;
            s.tb_log = tb_log;
        }
    }
    s.rows_per_block = s.nt ? 8 * s.nt : kPagedTcRows;
    s.grid = num_sms * (s.nt ? rows_ctas(c.head_dim, c.dtype, s.nt) : 1);
    if (s.nt == 0)
        while ((1LL << s.tb_log) < rows.max_rows && (2LL << s.tb_log) * group <= s.rows_per_block) ++s.tb_log;
    s.split = s.nt == 0 || positions > whole;
    s.spread = s.nt == 0 && blocks(s.tb_log) * kSpreadPieces < s.grid;
    return s;
}
size_t hdr_bytes(int grid) { return (static_cast<size_t>(2) * grid * sizeof(int4) + 255) & ~static_cast<size_t>(255); }

}  // namespace

size_t paged_attention_workspace(const PagedCacheDev& c, const PagedRowsDev& rows, int group, int num_sms) {
    // That of calls with fewer rows or sequences too: the shapes' needs are not quite in their order, and fewer blocks may be split.
    size_t need = 0;
    PagedRowsDev fewer = rows;
    const bool may_split = (static_cast<long long>(rows.table_width) << c.page_shift) > kWhole;
    for (int r = 1;; r = r < 32 && r + 1 < rows.max_rows ? r + 1 : rows.max_rows) {
        fewer.max_rows = std::min(r, rows.max_rows);
        const Shape s = shape_of(c, fewer, group, num_sms);
        const size_t bytes = hdr_bytes(s.grid) + static_cast<size_t>(2) * s.grid * s.rows_per_block * (c.head_dim + 2) * sizeof(float);
        if ((s.nt == 0 || may_split) && bytes > need) need = bytes;
        if (r >= rows.max_rows || s.nt == 0) return need;  // (the tcgen05 kernel needs the most)
    }
}

cudaError_t paged_attention_init() {
    cudaError_t e = rows_init_all<64, VERILLM_KV_BF16>();
    if (e == cudaSuccess) e = rows_init_all<64, VERILLM_KV_E4M3>();
    if (e == cudaSuccess) e = rows_init_all<64, VERILLM_KV_INT8>();
    if (e == cudaSuccess) e = rows_init_all<128, VERILLM_KV_BF16>();
    if (e == cudaSuccess) e = rows_init_all<128, VERILLM_KV_E4M3>();
    if (e == cudaSuccess) e = rows_init_all<128, VERILLM_KV_INT8>();
    if (e == cudaSuccess) e = paged_attention_tc_init();
    return e;
}

cudaError_t launch_paged_attention(PagedAttnParams p, void* workspace, int num_sms, cudaStream_t stream) {
    const Shape s = shape_of(p.c, p.r, p.group, num_sms);
    p.tb_log = s.tb_log;
    p.spread = s.spread ? 1 : 0;
    p.share_log = s.split ? PR_TILE_LOG : 30;
    p.hdr = s.split ? reinterpret_cast<int4*>(workspace) : nullptr;
    p.part = s.split ? reinterpret_cast<float*>(static_cast<char*>(workspace) + hdr_bytes(s.grid)) : nullptr;
    cudaError_t e = s.nt == 0              ? launch_paged_attention_tc(p, s.grid, stream)
                    : p.c.head_dim == 64 ? rows_launch_dtype<64>(p, s.nt, s.grid, stream)
                                         : rows_launch_dtype<128>(p, s.nt, s.grid, stream);
    if (e != cudaSuccess || !s.split) return e;
    cudaLaunchConfig_t cfg = {};
    const int rpw = s.nt ? 1 : 4;  // rows per warp of the join
    cfg.gridDim = dim3(s.grid, s.rows_per_block / (JOIN_WARPS * rpw));
    cfg.blockDim = dim3(JOIN_THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const bool narrow = p.c.head_dim == 64;
    void (*join)(PagedAttnParams, int) = s.nt ? (narrow ? paged_join_kernel<64, 1, true> : paged_join_kernel<128, 1, true>)
                                         : s.spread ? (narrow ? paged_join_kernel<64, 4, true> : paged_join_kernel<128, 4, true>)
                                                    : (narrow ? paged_join_kernel<64, 4, false> : paged_join_kernel<128, 4, false>);
    return cudaLaunchKernelEx(&cfg, join, p, s.rows_per_block);
}

}  // namespace vl
