// Causal grouped-query attention of new tokens over a paged cache, many rows per sequence (chunks of a prompt), on the
// fifth-generation tensor cores.  The same definition as the few-row kernel; here the products dominate.
//
// A block is up to 256 packed rows ((token, query head of the group), so that a kv head's keys and values serve all
// its query heads) of one (sequence, kv head), against tiles of 128 positions.  One CTA per SM holds the block as two
// groups of 128 rows; tensor memory is exactly full: per group 128 columns of scores and head_dim of output.
// While one group's four warps exponentiate a tile, the other group's products run.
//   warps 0-3, 4-7  softmax of the two groups, one row per thread: scores from tensor memory, running reference maximum
//                   and sum in registers, probabilities back as 16-bit pairs over the upper half of the score columns
//                   (three quarters first, so that most of P V runs under the last quarter's exponentials);
//                   they also write the results (and, 8-bit cache, scale the queries)
//   warps 8-11      bf16 cache: clean the values of tiles on the diagonal; 8-bit cache: widen the codes, half a tile at a
//                   time, and store them as operand tiles
//   warp 12         one thread issues S = Q K^T and O += P V of both groups (tcgen05.mma)
//   warp 13         walks the CTA's share of the work, hands the parts out and loads their queries (TMA)
//   warp 14         TMA loads of keys and values (8-bit cache: of codes into a ring of half tiles), a box and a lane per page
//   warp 15         8-bit cache: the scales of the next tiles
// The 64-column halves of all operand tiles use the 128-byte swizzle; values are consumed as they lie in memory
// ([key][dh], an MN-major B operand).
//
// 8-bit caches: codes are widened to fp16 operands with their scales in them, so that the softmax is the same as for
// bf16: an operand is code * scale / ref rounded once to fp16's 11 bits (bf16 keys and values have 8), with ref a
// power of two that brings the tile's largest scale into [2^6, 2^7): at most 448 * 2^7 fits.  The keys' ref multiplies the
// tile's scores; the values' ref is kept over the tiles of a block while it fits, and a larger one rescales the output.
// Queries are scaled row by row by a power of two into [1, 2), probabilities are taken 2^6 above the reference (up to
// 2^14), so that what fp16 cannot hold is below 2^-30 of the largest.  (Scales applied to the fp32 scores and
// probabilities instead cost the softmax two shared-memory reads and two products per four entries, which it had to wait
// for: 744 - 840 us for 1024 rows over 32768 positions.)
//
// Measured: 512 rows of each of 8 sequences over 4096 positions, 32 query heads on 8 of 128, bf16: 229 us = 986 TFLOP/s at full clock;
// 1024 rows over 32768, e4m3: 537 us = 1007 TFLOP/s, 570 - 580 at the power limit.  A step of both groups takes 3100 - 3200 cycles; the
// tensor pipe, the exp2 unit and shared memory need about 2048 of them each.
//
// Masked entries: scores are replaced by -inf.  Values behind the sequence's last position are whatever the page
// holds and become 0.  An infinite or NaN value (or value scale) in a tile that some rows may not see entirely is
// taken out of the product and put into the results of the rows that see it at the end ("stray").
#include "paged.cuh"

namespace vl {

namespace {

constexpr int PT_TILE_LOG = 7, PT_TILE = 1 << PT_TILE_LOG;
constexpr int PT_THREADS = 512;
constexpr int PT_GROUP_ROWS = 128, PT_ROWS = 2 * PT_GROUP_ROWS;
static_assert(PT_ROWS == kPagedTcRows, "");
constexpr int PT_KSTAGES = 2, PT_VSTAGES = 2, PT_SCALES = PT_KSTAGES + 1;
constexpr int PT_TMEM_COLS = 512;  // S of the groups at 0 and 128, O at 256 and 384
// The reference maximum is raised when a score exceeds it by pt_raise (log2), to the score less pt_lift.
constexpr float pt_raise(bool bf16) { return bf16 ? 8.f : 14.f; }
constexpr float pt_lift(bool bf16) { return bf16 ? 0.f : 6.f; }
// registers per thread of the roles; together what 512 threads are launched with (128 each)
constexpr int PT_REGS_SOFTMAX = 192, PT_REGS_OTHER = 64;
static_assert(2 * PT_REGS_SOFTMAX + 2 * PT_REGS_OTHER <= 4 * 128, "");
constexpr int PT_RAW = 3;  // half tiles of codes on their way

template <int DH, int DTYPE>
struct PtSmem {
    static constexpr bool BF16 = DTYPE == VERILLM_KV_BF16;
    static constexpr uint32_t Q_HALF = PT_ROWS * 128;  // 64 columns of all rows
    static constexpr uint32_t KV_HALF = PT_TILE * 128;
    static constexpr uint32_t KV_BYTES = KV_HALF * (DH / 64);
    static constexpr uint32_t K_OFF = Q_HALF * (DH / 64);
    static constexpr uint32_t V_OFF = K_OFF + PT_KSTAGES * KV_BYTES;
    static constexpr uint32_t SC_OFF = V_OFF + PT_VSTAGES * KV_BYTES;  // per slot: 128 key and 128 value scales, a word each
    static constexpr uint32_t SC_BYTES = 2 * PT_TILE * 4;
    static constexpr uint32_t RAW_OFF = SC_OFF + (BF16 ? 0 : PT_SCALES * SC_BYTES);
    static constexpr uint32_t RAW_BYTES = PT_TILE / 2 * DH;  // codes of half a tile
    static constexpr uint32_t BAR_OFF = RAW_OFF + (BF16 ? 0 : PT_RAW * RAW_BYTES);
    static constexpr uint32_t TOTAL = BAR_OFF + 640 + sizeof(ShareScratch);
};

// MN-major operand (V as stored: [key][dh]): 64 columns of a key are a row of 128 bytes, 8 keys per 1024-byte swizzle
// atom; `lbo_bytes` separates the 64-column halves.
__device__ __forceinline__ uint64_t pt_desc_mn(uint32_t tile_smem, uint32_t lbo_bytes) {
    const uint64_t lo = static_cast<uint64_t>((tile_smem & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(lbo_bytes >> 4) << 16);
    const uint64_t hi = static_cast<uint64_t>(1024u >> 4) | (1ull << 14) | (2ull << 29);
    return lo | (hi << 32);
}
// kind::f16 with fp32 accumulators; operands bf16 or fp16, B K-major or (mn) MN-major
__host__ __device__ constexpr uint32_t pt_idesc(bool bf16, int n, bool mn) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (mn ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) |
           (static_cast<uint32_t>(PT_GROUP_ROWS >> 4) << 24);
}
__device__ __forceinline__ float2 pt_fma2(float2 a, float2 b, float2 c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(d)
        : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
    return reinterpret_cast<float2&>(d);
}
__device__ __forceinline__ float2 pt_add2(float2 a, float2 b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
    return reinterpret_cast<float2&>(d);
}
__device__ __forceinline__ float pt_max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ void sts16(uint32_t addr, const uint4& x) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ void stg32(void* p, const uint32_t (&r)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
// Bounded wait of a whole warp, with one answer for all its lanes.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, int* status) {
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, status));
}
// The issuing warp runs converged, with operands in warp-uniform registers, and one elected lane issues: fewer
// instructions per product than a lone lane, whose operands have to be moved to uniform registers each time.
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(r));
    return r;
}
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader)
        : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t leader, uint32_t bar) {
    asm volatile(
        "{\n.reg .pred q;\nsetp.ne.b32 q, %1, 0;\n@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar), "r"(leader)
        : "memory");
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }
template <int N>
__device__ __forceinline__ void set_registers(bool more) {
    if (more) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// Four codes times a scale given as the sum of two fp16 numbers (both halves of sh, sl) -> fp16 pairs (0, 1) and (2, 3): code * sh +
// code * sl, rounded once to fp16 but for the rounding of the small second product.
template <int DTYPE>
__device__ __forceinline__ uint2 scaled4(uint32_t w, uint32_t sh, uint32_t sl) {
    const uint2 x = widen4_half<DTYPE>(w);
    uint2 y;
    asm("{\n.reg .b32 t;\nmul.rn.f16x2 t, %1, %3;\nfma.rn.f16x2 %0, %1, %2, t;\n}\n" : "=r"(y.x) : "r"(x.x), "r"(sh), "r"(sl));
    asm("{\n.reg .b32 t;\nmul.rn.f16x2 t, %1, %3;\nfma.rn.f16x2 %0, %1, %2, t;\n}\n" : "=r"(y.y) : "r"(x.y), "r"(sh), "r"(sl));
    return y;
}

__device__ __forceinline__ bool odd_bf16(uint32_t bits16) { return (bits16 & 0x7F80u) == 0x7F80u; }

// The part of a block that a CTA works on, as the roles see it.  One warp walks the CTA's share and hands the parts
// out through a small ring in shared memory, which keeps the walk out of everybody else's registers.
struct Part {
    int row0, first_pos, rows, seq;  // packed row of the first token, its position, packed rows (0: no more parts), sequence
    int kvh, t0, t1, whole;          // kv head, tiles, whether these are all of the block's
    __device__ __forceinline__ int end(int group) const { return first_pos + rows / group; }  // of the visible keys
    // first tile that some row may not see entirely: the tiles before it end at or before first_pos
    __device__ __forceinline__ int mask_tile() const { return first_pos < 0 ? 0 : (first_pos + 1) >> PT_TILE_LOG; }
};
constexpr int PT_PARTS = 4;  // ring of parts

// Which of the 32 columns from col0 on receive a NaN, +inf or -inf from values of keys [from, to) that are not finite.
struct Stray {
    uint32_t nan, pinf, ninf;
};
template <int DH, int DTYPE>
__device__ __noinline__ Stray find_stray(const PagedAttnParams& p, int seq, int kvh, int from, int to, int col0) {
    Stray x = {0u, 0u, 0u};
    for (int key = from; key < to; ++key) {
        const int page = load_page(p.r, p.c.page_shift, p.c.n_pages, seq, key, nullptr);
        const size_t vec = ((static_cast<size_t>(page) * p.c.n_kv_heads + kvh) << p.c.page_shift) + (key & ((1 << p.c.page_shift) - 1));
        if (DTYPE != VERILLM_KV_BF16) {
            if (!isfinite(p.c.v_scale[vec])) x.nan = 0xFFFFFFFFu;
            continue;
        }
        const unsigned short* v = reinterpret_cast<const unsigned short*>(p.c.v) + vec * DH + col0;
        for (int i = 0; i < 32; ++i) {
            const uint32_t b = v[i];
            if (!odd_bf16(b)) continue;
            if (b & 0x7Fu) x.nan |= 1u << i;
            else if (b & 0x8000u) x.ninf |= 1u << i;
            else x.pinf |= 1u << i;
        }
    }
    return x;
}

template <int DH, int DTYPE>
__global__ void __launch_bounds__(PT_THREADS, 1)
paged_tc_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                const __grid_constant__ PagedAttnParams p) {
    using L = PtSmem<DH, DTYPE>;
    constexpr bool BF16 = L::BF16;
    constexpr int HALVES = DH / 64;
    extern __shared__ __align__(1024) uint8_t pt_smem[];
    const uint32_t sbase = smem_u32(pt_smem);
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    if ((sbase & 1023u) != 0u) {  // the swizzled tiles need a 1024-byte aligned base
        if (tid == 0) {
            raise_status(p.status, VERILLM_DEV_WAIT_TIMEOUT);
            no_headers(p.hdr);
        }
        return;
    }
    const uint32_t q_s = sbase;
    auto k_s = [&](int b) { return sbase + L::K_OFF + b * L::KV_BYTES; };
    auto v_s = [&](int b) { return sbase + L::V_OFF + b * L::KV_BYTES; };
    const uint32_t bar = sbase + L::BAR_OFF;
    auto q_full = [&](int w) { return bar + 8 * w; };
    auto s_full = [&](int w) { return bar + 16 + 8 * w; };
    auto o_done = [&](int w) { return bar + 32 + 8 * w; };
    auto p_half = [&](int w, int h) { return bar + 48 + 16 * w + 8 * h; };
    auto k_full = [&](int b) { return bar + 80 + 8 * b; };
    auto k_empty = [&](int b) { return bar + 112 + 8 * b; };
    auto v_full = [&](int b) { return bar + 144 + 8 * b; };
    auto v_empty = [&](int b) { return bar + 176 + 8 * b; };
    auto sc_full = [&](int s) { return bar + 208 + 8 * s; };
    auto v_clean = [&](int b) { return bar + 232 + 8 * b; };
    auto part_full = [&](int i) { return bar + 248 + 8 * i; };
    auto part_empty = [&](int i) { return bar + 280 + 8 * i; };
    auto raw_full = [&](int i) { return bar + 312 + 8 * i; };
    auto raw_empty = [&](int i) { return bar + 336 + 8 * i; };
    auto word_full = [&](int i) { return bar + 360 + 8 * i; };
    auto word_empty = [&](int i) { return bar + 384 + 8 * i; };
    const uint32_t q_loaded = bar + 608, q_empty = bar + 616;
    auto q_ready = [&](int w) { return bar + 624 + 8 * w; };
    const uint32_t tmem_slot = bar + 408;
    volatile uint32_t* tmem_slot_ptr = reinterpret_cast<volatile uint32_t*>(pt_smem + L::BAR_OFF + 408);
    volatile int* failed = reinterpret_cast<volatile int*>(pt_smem + L::BAR_OFF + 412);
    volatile int* stray = reinterpret_cast<volatile int*>(pt_smem + L::BAR_OFF + 416);        // some value was taken out so far
    volatile float* sc_ref = reinterpret_cast<volatile float*>(pt_smem + L::BAR_OFF + 424);   // [PT_SCALES][2]: refs of a tile's keys and values
    volatile float* new_ref = reinterpret_cast<volatile float*>(pt_smem + L::BAR_OFF + 448);  // [PT_SCALES][2]: the same, beside the scale words
    int4* parts = reinterpret_cast<int4*>(pt_smem + L::BAR_OFF + 480);                        // [PT_PARTS][2]
    ShareScratch* scratch = reinterpret_cast<ShareScratch*>(pt_smem + L::BAR_OFF + 640);

    if (tid == 0) {
        *failed = 0;
        *stray = 0;
        mbar_init(q_loaded, 1);
        mbar_init(q_empty, 1);
        mbar_init(q_ready(0), 1);
        mbar_init(q_ready(1), 1);
        for (int w = 0; w < 2; ++w) {
            mbar_init(q_full(w), 4);
            mbar_init(s_full(w), 1);
            mbar_init(o_done(w), 1);
            mbar_init(p_half(w, 0), 4);
            mbar_init(p_half(w, 1), 4);
        }
        for (int b = 0; b < PT_KSTAGES; ++b) {
            mbar_init(k_full(b), BF16 ? 1 : 4);
            mbar_init(k_empty(b), 1);
        }
        for (int b = 0; b < PT_VSTAGES; ++b) {
            mbar_init(v_full(b), BF16 ? 1 : 4);
            mbar_init(v_empty(b), BF16 ? 1 + 4 : 1);  // the issuer; the cleaning warps
            mbar_init(v_clean(b), 4);
        }
        for (int s = 0; s < PT_SCALES; ++s) {
            mbar_init(sc_full(s), 1);
            mbar_init(word_full(s), 1);
            mbar_init(word_empty(s), 4);
        }
        for (int i = 0; i < PT_RAW; ++i) {
            mbar_init(raw_full(i), 1);
            mbar_init(raw_empty(i), 4);
        }
        for (int i = 0; i < PT_PARTS; ++i) {
            mbar_init(part_full(i), 1);
            mbar_init(part_empty(i), BF16 ? 14 : 15);  // one arrival per reading warp
        }
        fence_mbar_init();
    }
    if (warp == 12) {  // (under the reads below)
        tmem_alloc(tmem_slot, PT_TMEM_COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    WorkShare share;
    find_share(PT_TILE_LOG, p.r, p.c.page_shift, p.c.n_kv_heads, p.tb_log, PT_THREADS, scratch, share, p.status);
    pdl_launch_dependents();
    tc_fence_after();
    if (share.begin >= share.end) {
        if (tid == 0) no_headers(p.hdr);
        if (warp == 12) tmem_dealloc(*tmem_slot_ptr, PT_TMEM_COLS);
        return;
    }
    // All 512 columns are this CTA's, so they begin at 0 (known to the compiler); anything else is refused.
    constexpr uint32_t tmem_base = 0;
    const bool based = *tmem_slot_ptr == tmem_base;  // the same in all threads
    if (!based && tid == 0) {
        raise_status(p.status, VERILLM_DEV_WAIT_TIMEOUT);
        *failed = 1;
    }
    int* status = p.status;
    const int shift = p.c.page_shift, ps_mask = (1 << shift) - 1, n_kv = p.c.n_kv_heads, G = p.group;

    // Every role goes through the same parts; g counts the CTA's tiles (stage g % stages, phase g / stages).
    // take_part: the next part, read by whole warps; false at the end or when a wait gave up.
    auto take_part = [&](int& n, Part& u) -> bool {
        const int i = n % PT_PARTS;
        if (!warp_wait(part_full(i), (n / PT_PARTS) & 1, status)) {
            *failed = 1;
            return false;
        }
        const int4 a = parts[2 * i], b = parts[2 * i + 1];
        __syncwarp();
        if (lane == 0) mbar_arrive(part_empty(i));
        ++n;
        u.row0 = a.x; u.first_pos = a.y; u.rows = a.z; u.seq = a.w;
        u.kvh = b.x; u.t0 = b.y; u.t1 = b.z; u.whole = b.w;
        return u.rows != 0;
    };
    int np = 0;
    Part u;
    bool ok = based;

    if (!ok) {
    } else if (warp < 8) {
        // ------------------------------------------------------------ softmax, one row per thread
        set_registers<PT_REGS_SOFTMAX>(true);
        const int w = warp >> 2;
        const int r = tid;  // row of the block (the two groups' threads are 0 .. 255)
        const uint32_t lane_base = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        const uint32_t s_addr = lane_base + w * 128, o_addr = lane_base + 256 + w * 128;
        const float sl2 = rsqrtf(static_cast<float>(DH)) * kLog2e;
        int g = 0, sg = 0, au = 0;  // tiles of the CTA, tiles and parts of this group
        // the row's place in the current part: packed row, query head, last visible key
        bool valid = false;
        size_t row = 0;
        int hd = 0, pos = -1;
        float rf = sl2;  // factor of the scores in log2 units
        auto next_part = [&]() {  // the next part in which this group has rows
            while (take_part(np, u)) {
                if (w * PT_GROUP_ROWS < u.rows) return true;
                g += u.t1 - u.t0;
            }
            return false;
        };
        int nq = 0;  // parts of this group whose queries were awaited
        auto place = [&]() {
            valid = r < u.rows;
            const int tok = valid ? r / G : 0;
            hd = u.kvh * G + (valid ? r - tok * G : 0);
            row = static_cast<size_t>(u.row0 + tok);
            pos = valid ? u.first_pos + tok : -1;
        };
        // 8-bit pools: the row's queries to fp16, in place
        auto convert_q = [&]() -> bool {
            if (BF16) return true;
            if (!warp_wait(q_ready(w), nq++ & 1, status)) return false;
            uint4 qx[DH / 8];
            const uint32_t at = q_s + r * 128;
            uint32_t mx = 0;
#pragma unroll
            for (int c = 0; c < DH / 8; ++c) {
                qx[c] = lds16(at + (c >> 3) * L::Q_HALF + (((c & 7) ^ (r & 7)) << 4));
                mx = max(mx, abs_max8(qx[c]));
            }
            const uint32_t e = row_exponent(mx);
            const float down = __uint_as_float((254u - e) << 23);
            rf = sl2 * __uint_as_float(e << 23);
#pragma unroll
            for (int c = 0; c < DH / 8; ++c) {
                const uint4 x = qx[c];
                sts16(at + (c >> 3) * L::Q_HALF + (((c & 7) ^ (r & 7)) << 4),
                      make_uint4(pack_half(bf16_lo(x.x) * down, bf16_hi(x.x) * down), pack_half(bf16_lo(x.y) * down, bf16_hi(x.y) * down),
                                 pack_half(bf16_lo(x.z) * down, bf16_hi(x.z) * down), pack_half(bf16_lo(x.w) * down, bf16_hi(x.w) * down)));
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full(w));
            return true;
        };
        const bool wide_out = ((reinterpret_cast<uintptr_t>(p.out) | static_cast<uintptr_t>(p.out_stride * 2)) & 31u) == 0;
        bool have = next_part();
        if (have) {
            place();
            ok = convert_q();
        }
        while (have && ok) {
            const int mask_tile = u.mask_tile();
            float m_ref = -INFINITY, l_run = 0.f, vref = 0.f;
            for (int t = u.t0; t < u.t1; ++t, ++g, ++sg) {
                const int key0 = t << PT_TILE_LOG;
                const bool masked = t >= mask_tile;
                const int lim = pos - key0;  // visible: column <= lim
                if (!warp_wait(s_full(w), sg & 1, status)) { ok = false; break; }
                // (after the scores: a group that skipped blocks would misread the phase of a slot it has not reached;
                // now it has completed, and cannot complete again before this group's probabilities)
                if (!BF16 && !warp_wait(sc_full(g % PT_SCALES), (g / PT_SCALES) & 1, status)) { ok = false; break; }
                tc_fence_after();
                uint32_t v0[32], v1[32], v2[32], v3[32];
                float rt = rf, vnew = 0.f;
                if (!BF16) {
                    // not below the smallest normal number: 0 times a masked entry's -inf would be NaN (a score is
                    // below 2^24 before this factor, so none of those it concerns reaches 2^-100)
                    rt = fmaxf(rf * sc_ref[2 * (g % PT_SCALES)], 1.17549435e-38f);
                    vnew = sc_ref[2 * (g % PT_SCALES) + 1];
                }
                auto prepare = [&](uint32_t (&v)[32], int c) {  // masks the scores of columns [c, c + 32)
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c + i > lim) v[i] = 0xFF800000u;  // -inf
                    }
                };
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                tmem_ld32(s_addr, v0);
                tmem_ld32(s_addr + 32, v1);
                tmem_ld32(s_addr + 64, v2);
                tmem_ld32(s_addr + 96, v3);
                tmem_ld_wait_regs(v0);
                tmem_ld_wait_regs(v1);
                tmem_ld_wait_regs(v2);
                tmem_ld_wait_regs(v3);
                prepare(v0, 0);
                prepare(v1, 32);
                prepare(v2, 64);
                prepare(v3, 96);
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    mx4[i & 1] = pt_max3(mx4[i & 1], __uint_as_float(v0[i]), __uint_as_float(v1[i]));
                    mx4[2 + (i & 1)] = pt_max3(mx4[2 + (i & 1)], __uint_as_float(v2[i]), __uint_as_float(v3[i]));
                }
                const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * rt;
                const bool grow = valid && mx > m_ref + pt_raise(BF16);
                float corr = 1.f;
                bool fix = grow;
                if (!BF16 && vnew != vref) {  // the same in all threads
                    corr = vref / vnew;
                    vref = vnew;
                    fix = true;
                }
                if (__any_sync(0xFFFFFFFFu, fix)) {
                    if (grow) {
                        const float c = exp2_fast(m_ref - (mx - pt_lift(BF16)));
                        corr *= c;
                        l_run *= c;
                        m_ref = mx - pt_lift(BF16);
                    }
                    if (t != u.t0) {  // O holds the earlier tiles: this tile's scores were issued after their P V
#pragma unroll 1
                        for (int c = 0; c < DH / 32; ++c) {
                            uint32_t o[32];
                            tmem_ld32(o_addr + c * 32, o);
                            tmem_ld_wait_regs(o);
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
                            tmem_st32(o_addr + c * 32, o);
                        }
                        tmem_st_wait();
                    }
                }
                const float nm = m_ref == -INFINITY ? 0.f : -m_ref;
                const float2 nm2 = make_float2(nm, nm), rt2 = make_float2(rt, rt);
                float2 rs2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                // probabilities of columns [c, c + 32) as 16 packed columns over the upper half of the scores
                auto probabilities = [&](const uint32_t (&v)[32], int c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 x = pt_fma2(make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), rt2, nm2);
                        const float2 e = make_float2(exp2_fast(x.x), exp2_fast(x.y));
                        rs2[i & 1] = pt_add2(rs2[i & 1], e);
                        pk[i] = BF16 ? pack_bf16(e.x, e.y) : pack_half(e.x, e.y);
                    }
                    tmem_st16(s_addr + 64 + (c >> 1), pk);
                };
                auto deliver = [&](int h) {
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_half(w, h));
                };
                probabilities(v3, 96);
                probabilities(v2, 64);
                probabilities(v1, 32);
                deliver(0);
                probabilities(v0, 0);
                deliver(1);
                l_run += (rs2[0].x + rs2[0].y) + (rs2[1].x + rs2[1].y);
            }
            if (!ok) break;
            // ---- results: the whole block's, or this part's for the join.  The next part's queries are prepared first, so
            // that its first scores are formed under the output pass.
            const bool whole = u.whole != 0, row_valid = valid;
            const size_t out_row = row;
            const int out_hd = hd, seq = u.seq, kvh = u.kvh;
            const int odd_from = max(u.t0, mask_tile) << PT_TILE_LOG, odd_to = min(pos + 1, u.t1 << PT_TILE_LOG);
            float* part = part_slot(p.part, 2 * static_cast<int>(blockIdx.x) + (u.t0 == 0 ? 1 : 0), PT_ROWS, DH);
            have = next_part();
            if (have) place();
            if (have && !convert_q()) { ok = false; break; }
            if (!warp_wait(o_done(w), au & 1, status)) { ok = false; break; }
            ++au;
            tc_fence_after();
            const float inv = (whole ? (l_run == 0.f ? 0.f : 1.f / l_run) : 1.f) * (BF16 ? 1.f : vref);
            const bool odd = *stray != 0;
            if (row_valid) {
                if (whole) {
                    if (p.lse) p.lse[out_row * p.n_heads + out_hd] = l_run == 0.f ? -INFINITY : m_ref * kLn2 + logf(l_run);
                } else {
                    part[r] = m_ref;
                    part[PT_ROWS + r] = l_run;
                }
            }
            uint32_t oo[DH / 32][32];  // all at once: one latency
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) tmem_ld32(o_addr + c * 32, oo[c]);
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) tmem_ld_wait_regs(oo[c]);
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) {
                uint32_t(&o)[32] = oo[c];
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = l_run == 0.f ? 0u : __float_as_uint(__uint_as_float(o[i]) * inv);
                if (odd) {
                    const Stray x = find_stray<DH, DTYPE>(p, seq, kvh, odd_from, odd_to, c * 32);
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        if ((x.nan >> i) & 1u) o[i] = 0x7FC00000u;
                        if ((x.pinf >> i) & 1u) o[i] = __float_as_uint(__uint_as_float(o[i]) + INFINITY);
                        if ((x.ninf >> i) & 1u) o[i] = __float_as_uint(__uint_as_float(o[i]) - INFINITY);
                    }
                }
                if (row_valid && whole) {
                    __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.out) + out_row * p.out_stride + static_cast<size_t>(out_hd) * DH + c * 32;
                    uint32_t y[2][8];
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i >> 3][i & 7] = pack_bf16(__uint_as_float(o[2 * i]), __uint_as_float(o[2 * i + 1]));
                    if (wide_out) {
                        stg32(dst, y[0]);
                        stg32(dst + 16, y[1]);
                    } else {
#pragma unroll
                        for (int h = 0; h < 4; ++h)
                            reinterpret_cast<uint4*>(dst)[h] = make_uint4(y[h >> 1][4 * (h & 1)], y[h >> 1][4 * (h & 1) + 1], y[h >> 1][4 * (h & 1) + 2], y[h >> 1][4 * (h & 1) + 3]);
                    }
                } else if (row_valid) {
                    float* dst = part + 2 * PT_ROWS + r * DH + c * 32;
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        uint32_t y[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = o[8 * h + i];
                        stg32(dst + 8 * h, y);
                    }
                }
                __syncwarp();
            }
        }
    } else if (warp < 12) {
        set_registers<PT_REGS_OTHER>(false);
        const int ht = tid - 256;  // thread of the helper group
        int g = 0;
        if (BF16) {
            // ------------------------------------------------------------ clean the values of masked tiles
            while (ok && take_part(np, u)) {
                const int mask_tile = u.mask_tile(), end = u.end(G);
                for (int t = u.t0; t < u.t1; ++t, ++g) {
                    // every tile is awaited and released here too, masked or not: a phase parity says nothing to a
                    // thread that skipped phases
                    if (!warp_wait(v_full(g % PT_VSTAGES), (g / PT_VSTAGES) & 1, status)) { ok = false; break; }
                    if (t < mask_tile) {
                        if (lane == 0) mbar_arrive(v_empty(g % PT_VSTAGES));
                        continue;
                    }
                    const uint32_t row = v_s(g % PT_VSTAGES) + ht * 128;
                    const bool gone = (t << PT_TILE_LOG) + ht >= end;
                    bool found = false;
#pragma unroll
                    for (int h = 0; h < HALVES; ++h)
#pragma unroll 2
                        for (int c = 0; c < 8; ++c) {
                            const uint32_t a = row + h * L::KV_HALF + ((c ^ (ht & 7)) << 4);
                            if (gone) {
                                sts16(a, make_uint4(0u, 0u, 0u, 0u));
                                continue;
                            }
                            const uint4 x = lds16(a);
                            const uint32_t m = __vmaxu2(__vmaxu2(x.x & 0x7F807F80u, x.y & 0x7F807F80u), __vmaxu2(x.z & 0x7F807F80u, x.w & 0x7F807F80u));
                            if (!odd_bf16(m) && !odd_bf16(m >> 16)) continue;
                            found = true;
                            uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if (odd_bf16(y[i])) y[i] &= 0xFFFF0000u;
                                if (odd_bf16(y[i] >> 16)) y[i] &= 0x0000FFFFu;
                            }
                            sts16(a, make_uint4(y[0], y[1], y[2], y[3]));
                        }
                    if (found) *stray = 1;
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(v_clean(g % PT_VSTAGES));
                        mbar_arrive(v_empty(g % PT_VSTAGES));
                    }
                }
            }
        } else {
            // ------------------------------------------------------------ widen the codes, half a tile at a time
            constexpr int CPR = DH / 16;             // 16-byte pieces of a vector
            constexpr int RPP = 128 / CPR;           // rows per pass over the 128 threads
            constexpr int NP = (PT_TILE / 2) / RPP;  // passes per half tile
            const int c = ht % CPR, r0 = ht / CPR;
            int n = 0;  // half tiles so far
            while (ok && take_part(np, u)) {
                const int end = u.end(G);
                for (int t = u.t0; t < u.t1 && ok; ++t, ++g) {
                    const int kb = g % PT_KSTAGES, vb = g % PT_VSTAGES, slot = g % PT_SCALES;
                    const int left = end - (t << PT_TILE_LOG);  // visible keys from the tile's first on
                    const uint32_t words = sbase + L::SC_OFF + slot * L::SC_BYTES;
#pragma unroll 1
                    for (int q = 0; q < 4; ++q, ++n) {  // keys 0 - 63, 64 - 127, values 0 - 63, 64 - 127
                        if (q == 0) {
                            if (g >= PT_KSTAGES && !warp_wait(k_empty(kb), ((g / PT_KSTAGES) - 1) & 1, status)) { ok = false; break; }
                            if (!warp_wait(word_full(slot), (g / PT_SCALES) & 1, status)) { ok = false; break; }
                            // The refs go on to the softmax in a ring of their own: its slot's previous ones belong to tile
                            // g - KSTAGES - 1, whose probabilities preceded the product that freed this key stage.
                            if (warp == 8 && lane == 0) {
                                sc_ref[2 * slot] = new_ref[2 * slot];
                                sc_ref[2 * slot + 1] = new_ref[2 * slot + 1];
                                mbar_arrive(sc_full(slot));
                            }
                        } else if (q == 2) {
                            if (g >= PT_VSTAGES && !warp_wait(v_empty(vb), ((g / PT_VSTAGES) - 1) & 1, status)) { ok = false; break; }
                        }
                        if (!warp_wait(raw_full(n % PT_RAW), (n / PT_RAW) & 1, status)) { ok = false; break; }
                        const uint32_t src = sbase + L::RAW_OFF + (n % PT_RAW) * L::RAW_BYTES + ht * 16;
                        const uint32_t dst = (q < 2 ? k_s(kb) : v_s(vb)) + (c >> 2) * L::KV_HALF;
                        const uint32_t ws = words + (q < 2 ? 0 : PT_TILE * 4);
                        uint4 x[NP];
                        uint32_t sw[NP];
#pragma unroll
                        for (int i = 0; i < NP; ++i) {
                            x[i] = lds16(src + i * 2048);
                            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(sw[i]) : "r"(ws + ((q & 1) * (PT_TILE / 2) + i * RPP + r0) * 4) : "memory");
                        }
                        if (left < PT_TILE) {  // codes behind the last key are whatever the page holds, NaN codes too
#pragma unroll
                            for (int i = 0; i < NP; ++i)
                                if ((q & 1) * (PT_TILE / 2) + i * RPP + r0 >= left) x[i] = make_uint4(0u, 0u, 0u, 0u);
                        }
#pragma unroll
                        for (int i = 0; i < NP; ++i) {
                            const int row = (q & 1) * (PT_TILE / 2) + i * RPP + r0;
                            const uint32_t sh = __byte_perm(sw[i], 0u, 0x1010), sl = __byte_perm(sw[i], 0u, 0x3232);
                            const uint2 a = scaled4<DTYPE>(x[i].x, sh, sl), b = scaled4<DTYPE>(x[i].y, sh, sl), d = scaled4<DTYPE>(x[i].z, sh, sl), e = scaled4<DTYPE>(x[i].w, sh, sl);
                            // the lanes of the second half store their pieces in the other order: 8 lanes then reach all banks
                            const int c16 = 2 * (c & 3), odd = c >> 2;
                            const uint4 lo = make_uint4(a.x, a.y, b.x, b.y), hi = make_uint4(d.x, d.y, e.x, e.y);
                            sts16(dst + row * 128 + (((c16 + odd) ^ (row & 7)) << 4), odd ? hi : lo);
                            sts16(dst + row * 128 + (((c16 + 1 - odd) ^ (row & 7)) << 4), odd ? lo : hi);
                        }
                        if (q & 1) fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(raw_empty(n % PT_RAW));
                            if (q == 1) mbar_arrive(k_full(kb));
                            if (q == 3) {
                                mbar_arrive(v_full(vb));
                                mbar_arrive(word_empty(slot));
                            }
                        }
                    }
                }
            }
        }
    } else {
        set_registers<PT_REGS_OTHER>(false);
        if (warp == 12) {
        // ------------------------------------------------------------ product issuer (one warp)
        // One warp issues for both groups, P V of a tile and Q K^T of the next back to back, group after group: the
        // groups then work in opposite phases, one on its exponentials while the other's products run.  (With an issuer
        // per group the two fell into step: both waited for the products, then both for the exponentials.)
        {
            constexpr uint32_t idesc_s = pt_idesc(BF16, PT_TILE, false), idesc_o = pt_idesc(BF16, DH, true);
            const uint64_t q_desc = umma_desc_k_sw128(q_s);
            const uint32_t leader = elect_one();
            int g = 0, sg[2] = {0, 0}, au[2] = {0, 0};  // tiles of the CTA; tiles and blocks of each group
            uint32_t clean = 0;                         // phase of each value stage's cleaning
            while (take_part(np, u)) {
                const int mask_tile = uniform(u.mask_tile()), t0 = uniform(u.t0), t1 = uniform(u.t1);
                const int groups = uniform(u.rows) > PT_GROUP_ROWS ? 2 : 1;
                auto scores = [&](int w, int gt) {  // S of group w = Q K^T of the CTA's tile gt
                    const uint32_t s_tmem = w * 128;
                    const uint64_t qd = q_desc + static_cast<uint64_t>(w * ((PT_GROUP_ROWS * 128) >> 4));
                    const uint64_t kd = umma_desc_k_sw128(k_s(gt % PT_KSTAGES));
#pragma unroll
                    for (int s = 0; s < DH / 16; ++s)
                        mma_ss(leader, s_tmem, qd + static_cast<uint64_t>((s / 4) * (L::Q_HALF >> 4) + 2 * (s % 4)),
                                  kd + static_cast<uint64_t>((s / 4) * (L::KV_HALF >> 4) + 2 * (s % 4)), idesc_s, s != 0 ? 1u : 0u);
                    mma_commit(leader, s_full(w));
                };
                if (!warp_wait(k_full(g % PT_KSTAGES), (g / PT_KSTAGES) & 1, status)) { ok = false; break; }
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    if (w >= groups) break;
                    if (!warp_wait(BF16 ? q_loaded : q_full(w), (BF16 ? np - 1 : au[w]) & 1, status)) { ok = false; break; }
                    tc_fence_after();
                    scores(w, g);
                    ++au[w];
                }
                if (!ok) break;
                mma_commit(leader, k_empty(g % PT_KSTAGES));
                if (t0 + 1 == t1) mma_commit(leader, q_empty);
                for (int t = t0; t < t1; ++t, ++g) {
                    const int vb = g % PT_VSTAGES;
                    const bool more = t + 1 < t1;
                    if (!warp_wait(v_full(vb), (g / PT_VSTAGES) & 1, status)) { ok = false; break; }
                    if (BF16 && t >= mask_tile) {
                        if (!warp_wait(v_clean(vb), (clean >> vb) & 1u, status)) { ok = false; break; }
                        clean ^= 1u << vb;
                    }
                    if (more && !warp_wait(k_full((g + 1) % PT_KSTAGES), ((g + 1) / PT_KSTAGES) & 1, status)) { ok = false; break; }
                    const uint64_t vd = pt_desc_mn(v_s(vb), L::KV_HALF);
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        if (w >= groups) break;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {  // keys 32 - 127 first
                            if (!warp_wait(p_half(w, h), sg[w] & 1, status)) { ok = false; break; }
                            tc_fence_after();
#pragma unroll
                            for (int i = 0; i < (h == 0 ? 6 : 2); ++i) {
                                const int s = (h == 0 ? 2 : 0) + i;
                                mma_ts(leader, 256 + w * 128, w * 128 + 64 + s * 8, vd + static_cast<uint64_t>(s * (2048 >> 4)), idesc_o,
                                             t == t0 && h == 0 && i == 0 ? 0u : 1u);
                            }
                        }
                        if (!ok) break;
                        ++sg[w];
                        if (more) scores(w, g + 1);
                        else mma_commit(leader, o_done(w));
                    }
                    if (!ok) break;
                    mma_commit(leader, v_empty(vb));
                    if (more) mma_commit(leader, k_empty((g + 1) % PT_KSTAGES));
                    if (t + 2 == t1) mma_commit(leader, q_empty);  // the part's last scores are under way
                }
                if (!ok) break;
            }
        }
        } else if (BF16 && warp == 14) {
        // ------------------------------------------------------------ TMA producer: one box per page, a lane each
        const int bp = min(1 << shift, PT_TILE);  // positions per box
        int g = 0;
        while (ok && take_part(np, u)) {
            const int end = u.end(G);
            for (int t = u.t0; t < u.t1; ++t, ++g) {
                const int kb = g % PT_KSTAGES, vb = g % PT_VSTAGES;
                const int left = end - (t << PT_TILE_LOG);
                const int boxes = left <= 0 ? 0 : (min(left, PT_TILE) + bp - 1) / bp;
                int y = 0;
                if (lane < boxes) {
                    const int key = (t << PT_TILE_LOG) + lane * bp;
                    y = ((load_page(p.r, shift, p.c.n_pages, u.seq, key, status) * n_kv + u.kvh) << shift) + (key & ps_mask);
                }
                if (g >= PT_KSTAGES && !warp_wait(k_empty(kb), ((g / PT_KSTAGES) - 1) & 1, status)) { ok = false; break; }
                if (lane == 0) mbar_arrive_expect_tx(k_full(kb), boxes * bp * DH * 2);
                __syncwarp();
                if (lane < boxes)
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) tma_load_2d(k_s(kb) + h * L::KV_HALF + lane * bp * 128, &tmap_k, h * 64, y, k_full(kb));
                if (g >= PT_VSTAGES && !warp_wait(v_empty(vb), ((g / PT_VSTAGES) - 1) & 1, status)) { ok = false; break; }
                if (lane == 0) mbar_arrive_expect_tx(v_full(vb), boxes * bp * DH * 2);
                __syncwarp();
                if (lane < boxes)
#pragma unroll
                    for (int h = 0; h < HALVES; ++h) tma_load_2d(v_s(vb) + h * L::KV_HALF + lane * bp * 128, &tmap_v, h * 64, y, v_full(vb));
            }
        }
        } else if (!BF16 && warp == 14) {
        // ------------------------------------------------------------ TMA producer of codes: half tiles, a box per page
        const int bp = min(1 << shift, PT_TILE / 2), per_half = (PT_TILE / 2) / bp;
        int n = 0;
        while (ok && take_part(np, u)) {
            const int end = u.end(G);
            for (int t = u.t0; t < u.t1 && ok; ++t) {
                const int key = (t << PT_TILE_LOG) + lane * bp;  // lanes 0 .. 2 per_half - 1
                const bool live = lane < 2 * per_half && key < end;
                const int y = live ? ((load_page(p.r, shift, p.c.n_pages, u.seq, key, status) * n_kv + u.kvh) << shift) + (key & ps_mask) : 0;
                const int boxes = __popc(__ballot_sync(0xFFFFFFFFu, live));
#pragma unroll 1
                for (int q = 0; q < 4; ++q, ++n) {
                    const int slot = n % PT_RAW, h = q & 1;
                    if (n >= PT_RAW && !warp_wait(raw_empty(slot), ((n / PT_RAW) - 1) & 1, status)) { ok = false; break; }
                    if (lane == 0) mbar_arrive_expect_tx(raw_full(slot), min(max(boxes - h * per_half, 0), per_half) * bp * DH);
                    __syncwarp();
                    if (live && lane / per_half == h)
                        tma_load_2d(sbase + L::RAW_OFF + slot * L::RAW_BYTES + (lane - h * per_half) * bp * DH, q < 2 ? &tmap_k : &tmap_v, 0, y, raw_full(slot));
                }
            }
        }
        } else if (!BF16 && warp == 15) {
        // ------------------------------------------------------------ scales of a tile: refs, and a word per key and value
        int g = 0;
        while (ok && take_part(np, u)) {
            const int end = u.end(G), mask_tile = u.mask_tile();
            float vref = 0.f;
            for (int t = u.t0; t < u.t1; ++t, ++g) {
                const int slot = g % PT_SCALES;
                const int key = (t << PT_TILE_LOG) + 4 * lane;
                float kq[4] = {0.f, 0.f, 0.f, 0.f}, vq[4] = {0.f, 0.f, 0.f, 0.f}, km = 0.f, vm = 0.f;
                if (key < end) {
                    const int page = load_page(p.r, shift, p.c.n_pages, u.seq, key, status);
                    const size_t vec = ((static_cast<size_t>(page) * n_kv + u.kvh) << shift) + (key & ps_mask);
                    const float4 a = __ldg(reinterpret_cast<const float4*>(p.c.k_scale + vec)), b = __ldg(reinterpret_cast<const float4*>(p.c.v_scale + vec));
                    kq[0] = a.x; kq[1] = a.y; kq[2] = a.z; kq[3] = a.w;
                    vq[0] = b.x; vq[1] = b.y; vq[2] = b.z; vq[3] = b.w;
#pragma unroll
                    for (int i = 1; i < 4; ++i)
                        if (key + i >= end) kq[i] = vq[i] = 0.f;  // behind the last key: whatever the page holds
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (t >= mask_tile && !isfinite(vq[i])) {
                        *stray = 1;
                        vq[i] = 0.f;
                    }
                    km = isfinite(kq[i]) ? fmaxf(km, kq[i]) : km;
                    vm = isfinite(vq[i]) ? fmaxf(vm, vq[i]) : vm;
                }
                const float kref = scale_ref(warp_max(km));
                if (__any_sync(0xFFFFFFFFu, vref == 0.f || vm > vref * kScaleRefMax)) vref = fmaxf(vref, scale_ref(warp_max(vm)));
                // scale / ref as the sum of two fp16 numbers
                const float kup = 1.f / kref, vup = 1.f / vref;  // powers of two, at most 2^126
                uint32_t kw[4], vw[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float kx = kq[i] * kup, vx = vq[i] * vup;
                    const float kh = __half2float(__float2half_rn(kx)), vh = __half2float(__float2half_rn(vx));
                    kw[i] = pack_half(kh, kx - kh);
                    vw[i] = pack_half(vh, vx - vh);
                }
                if (g >= PT_SCALES && !warp_wait(word_empty(slot), ((g / PT_SCALES) - 1) & 1, status)) { ok = false; break; }
                const uint32_t words = sbase + L::SC_OFF + slot * L::SC_BYTES + lane * 16;
                sts16(words, make_uint4(kw[0], kw[1], kw[2], kw[3]));
                sts16(words + PT_TILE * 4, make_uint4(vw[0], vw[1], vw[2], vw[3]));
                if (lane == 0) {
                    new_ref[2 * slot] = kref;
                    new_ref[2 * slot + 1] = vref;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(word_full(slot));
            }
        }
        } else if (warp == 13) {
        // ------------------------------------------------------------ hands out the parts
        BlockWalk k;
        walk_begin(PT_TILE_LOG, p.r, shift, p.tb_log, share, k);
        int4 header = make_int4(0, 0, 0, 0);
        if (p.spread && lane == 0) first_header(p.hdr, share, k);
        bool more = true;
        for (int n = 0; ok; ++n) {
            const int i = n % PT_PARTS;
            if (n >= PT_PARTS && !warp_wait(part_empty(i), ((n / PT_PARTS) - 1) & 1, status)) { ok = false; break; }
            if (more) {
                const int tok0 = k.j << p.tb_log;
                const bool whole = k.t0 == 0 && k.t1 == k.tiles;
                if (!whole && k.t0 == 0)
                    header = make_int4(last_cta(share, k) - static_cast<int>(blockIdx.x) + 1, k.seq, k.kvh, k.j);
                if (lane == 0) {
                    parts[2 * i] = make_int4(k.s.row0 + tok0, k.s.len - k.s.n + tok0, min(1 << p.tb_log, k.s.n - tok0) * G, k.seq);
                    parts[2 * i + 1] = make_int4(k.kvh, k.t0, k.t1, whole ? 1 : 0);
                }
            } else if (lane == 0) {
                parts[2 * i] = make_int4(0, 0, 0, 0);
                parts[2 * i + 1] = make_int4(0, 0, 0, 0);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(part_full(i));
            if (!more) break;
            // the part's queries, one box of (64 columns, heads of the group, tokens of a block) per half, once the
            // previous part's last scores are formed; rows behind the part's are other rows of q or zeros
            if (n > 0 && !warp_wait(q_empty, (n - 1) & 1, status)) { ok = false; break; }
            if (lane == 0) {
                mbar_arrive_expect_tx(q_loaded, static_cast<uint32_t>(G << p.tb_log) * DH * 2);
#pragma unroll
                for (int h = 0; h < HALVES; ++h) tma_load_3d(q_s + h * L::Q_HALF, &tmap_q, h * 64, k.kvh * G, k.s.row0 + (k.j << p.tb_log), q_loaded);
            }
            __syncwarp();
            if (!BF16) {  // passed on to the groups that have rows: a group that skips parts would misread q_loaded's phase
                if (!warp_wait(q_loaded, n & 1, status)) { ok = false; break; }
                if (lane == 0) {
                    mbar_arrive(q_ready(0));
                    if (min(1 << p.tb_log, k.s.n - (k.j << p.tb_log)) * G > PT_GROUP_ROWS) mbar_arrive(q_ready(1));
                }
                __syncwarp();
            }
            more = walk_next(PT_TILE_LOG, p.r, shift, n_kv, p.tb_log, share, k);
        }
        if (lane == 0) p.hdr[2 * blockIdx.x] = header;
        }
    }
    if (!ok) *failed = 1;

    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*failed) {
        if (tid == 0) no_headers(p.hdr);
        const long long t0 = clock64();  // let copies and products in flight land
        while (clock64() - t0 < 2000000LL) {
        }
        __syncthreads();
    }
    if (warp == 12) {
        tc_fence_after();
        tmem_dealloc(*tmem_slot_ptr, PT_TMEM_COLS);
    }
}

template <int DH, int DTYPE>
cudaError_t tc_init() {
    return cudaFuncSetAttribute(paged_tc_kernel<DH, DTYPE>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(PtSmem<DH, DTYPE>::TOTAL));
}
template <int DH, int DTYPE>
cudaError_t tc_launch(const PagedAttnParams& p, int grid, cudaStream_t stream) {
    CUtensorMap tq, tk, tv;
    if (make_tmap_bf16_heads(&tq, p.q, static_cast<uint64_t>(p.r.n_rows), static_cast<uint64_t>(p.n_heads), DH, static_cast<uint64_t>(p.q_stride),
                             static_cast<uint32_t>(p.group), 1u << p.tb_log) != 0)
        return cudaErrorInvalidValue;
    const uint64_t rows = static_cast<uint64_t>(p.c.n_pages) * p.c.n_kv_heads << p.c.page_shift;
    const uint32_t page = 1u << p.c.page_shift;
    if (DTYPE == VERILLM_KV_BF16) {
        const uint32_t box = page < PT_TILE ? page : PT_TILE;
        if (make_tmap_bf16_2d(&tk, p.c.k, rows, DH, DH, box) != 0 || make_tmap_bf16_2d(&tv, p.c.v, rows, DH, DH, box) != 0) return cudaErrorInvalidValue;
    } else {
        const uint32_t box = page < PT_TILE / 2 ? page : PT_TILE / 2;
        if (make_tmap_bytes_2d(&tk, p.c.k, rows, DH, box) != 0 || make_tmap_bytes_2d(&tv, p.c.v, rows, DH, box) != 0) return cudaErrorInvalidValue;
    }
    paged_tc_kernel<DH, DTYPE><<<grid, PT_THREADS, PtSmem<DH, DTYPE>::TOTAL, stream>>>(tq, tk, tv, p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t paged_attention_tc_init() {
    cudaError_t e = tc_init<64, VERILLM_KV_BF16>();
    if (e == cudaSuccess) e = tc_init<64, VERILLM_KV_E4M3>();
    if (e == cudaSuccess) e = tc_init<64, VERILLM_KV_INT8>();
    if (e == cudaSuccess) e = tc_init<128, VERILLM_KV_BF16>();
    if (e == cudaSuccess) e = tc_init<128, VERILLM_KV_E4M3>();
    if (e == cudaSuccess) e = tc_init<128, VERILLM_KV_INT8>();
    return e;
}

cudaError_t launch_paged_attention_tc(const PagedAttnParams& p, int grid, cudaStream_t stream) {
    const bool wide = p.c.head_dim == 128;
    if (p.c.dtype == VERILLM_KV_BF16) return wide ? tc_launch<128, VERILLM_KV_BF16>(p, grid, stream) : tc_launch<64, VERILLM_KV_BF16>(p, grid, stream);
    if (p.c.dtype == VERILLM_KV_E4M3) return wide ? tc_launch<128, VERILLM_KV_E4M3>(p, grid, stream) : tc_launch<64, VERILLM_KV_E4M3>(p, grid, stream);
    return wide ? tc_launch<128, VERILLM_KV_INT8>(p, grid, stream) : tc_launch<64, VERILLM_KV_INT8>(p, grid, stream);
}

}  // namespace vl
