// Products with 4-bit weights for more rows of x than a decode step's few (w4.cu has the definition and the kernel for those), and for any length.
//
// A CTA takes 128 outputs, up to 64 rows of x (more in further CTAs, which find the weights in L2) and a slice of the inputs, in units of 128:
// 8 KB of codes come by TMA, a warp group turns each output's codes into bf16 whole numbers (exact) and stores them into tensor memory as the
// first operand, lane = output; x comes by TMA as the second.  tcgen05 products of one scale group go to one of two accumulators in tensor memory;
// another warp group reads each, multiplies by its output's scale and adds to fp32 sums in registers.  So products are exact, scales are
// applied in fp32, and no weight is rounded again.  Slices of one tile are joined through the cluster's shared memory in the order of the inputs.
//
// What bounds it: the hand-overs.  A unit passes four roles (widened, multiplied, read out, its buffers free again), each 100 - 250 cycles behind the
// one before; a CTA keeps two units under way and takes about 860 cycles for each with the work itself left out, 1500 with it, and two CTAs share an SM.
// 64 rows x 28672 x 4096: 34.5 us = 435 TFLOP/s (floor 9.4 us, the codes' bytes); 16 rows 27.5 us; 64 rows x 4096 x 14336 in groups of 64 22 us.
// Tried: operands handed over by halves of units, twice as many under way (64 rows 0.3 us less, 16 rows 1.4 more), one CTA per SM over an equal share
// of all units with partial tiles in global memory (46 us and 6 for the join), tiles beginning at different inputs and scales prefetched into L2
// (no change), one issuing warp (no change).  What the outputs' stores and the slices' join cost counts too: with y written row by row behind each
// row's residual, and a join that only a part of the threads took part in, the first of these took 39 us and 64 rows x 9472 x 4096 33.5 instead of 20.
#include "common.cuh"
#include "kernels.h"

namespace vl {

namespace {

typedef __nv_bfloat16 bf16;

// warps 0-3 widen even units, 4-7 odd ones, 8-11 add up, 12 and 15 issue products, 13 loads x, 14 codes; two CTAs per SM
constexpr int T_THREADS = 512;
constexpr int T_REGS_WIDEN = 56, T_REGS_SUM = 104, T_REGS_REST = 40;  // 64 per thread at launch: 8 * 56 + 4 * 104 + 4 * 40 = 16 * 64
constexpr int T_TILE = 128;         // outputs per CTA
constexpr int T_UNIT = 128;         // inputs per unit
constexpr int T_WSTAGES = 3;        // stages of 2 units of codes: 128 rows of 128 bytes
constexpr int T_WBYTES = T_TILE * 128;
constexpr int T_XSTAGES = 4;
constexpr int T_ACOLS = T_UNIT / 2; // columns of one operand buffer
constexpr int T_DBUFS = 2;          // accumulators
constexpr int T_RING = 8;           // barriers of completed groups and units: twice what is under way, for whoever looks at every other one
constexpr int T_TMEM = 256;         // columns: two operand buffers and the accumulators

template <int N>
struct TcLayout {
    static constexpr int XBYTES = N * T_UNIT * 2, XHALF = XBYTES / 2;  // a stage of x: two boxes of N rows of 128 bytes
    static constexpr int X0 = T_WSTAGES * T_WBYTES, BARS = X0 + T_XSTAGES * XBYTES;
    static constexpr int W_FULL = 0, W_EMPTY = W_FULL + T_WSTAGES, U_FULL = W_EMPTY + T_WSTAGES, D_FULL = U_FULL + T_XSTAGES,
                         D_EMPTY = D_FULL + T_RING, U_DONE = D_EMPTY + T_RING, DRAIN = U_DONE + T_RING, N_BARS = DRAIN + 1;
    static constexpr int BYTES = BARS + N_BARS * 8 + 16;
};

__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(r));
    return r;
}
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader)
        : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t leader, uint32_t bar) {
    asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %1, 0;\n@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar), "r"(leader)
                 : "memory");
}
template <int N>
__device__ __forceinline__ void set_registers(bool more) {
    if (more) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, int* status) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, status)); }

// Position in a ring of barriers, and the phase there.
template <int LEN>
struct Ring {
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++at == LEN) {
            at = 0;
            phase ^= 1u;
        }
    }
};

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}

// The eight codes of a word as four pairs of bf16, in order: 0x4300 | u is 128 + u, less 136 is the code.
__device__ __forceinline__ void widen(uint32_t q, uint32_t* r) {
    const uint32_t t = q >> 4;
    const uint32_t m[4] = {__byte_perm(q, t, 0x4400), __byte_perm(q, t, 0x5511), __byte_perm(q, t, 0x6622), __byte_perm(q, t, 0x7733)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // (the compiler makes two instructions of an and and an or with constants)
        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r[i]) : "r"(m[i]), "r"(0x000F000Fu), "r"(0x43004300u));
        asm("sub.rn.bf16x2 %0, %0, %1;" : "+r"(r[i]) : "r"(0x43084308u));
    }
}

// Stores COUNT neighbours of y from (row, n) on, along a row or down a column, of which `live` exist.  What is added is read first: the reads wait
// together, and for no store.
template <int COUNT>
__device__ __forceinline__ void tc_store_y(const W4Params& p, int row, int n, bool along, const float* v, int live) {
    float r[COUNT];
    const long long ys = along ? 1 : p.y_stride;
    if (p.residual) {
        const float* res = p.residual + row * p.res_stride + n;
        const long long rs = along ? 1 : p.res_stride;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) r[i] = i < live ? res[i * rs] : 0.f;
#pragma unroll
        for (int i = 0; i < COUNT; ++i) r[i] += v[i];
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) r[i] = v[i];
    }
    if (p.out_f32) {
        float* y = reinterpret_cast<float*>(p.y) + row * p.y_stride + n;
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            if (i < live) y[i * ys] = r[i];
    } else {
        bf16* y = reinterpret_cast<bf16*>(p.y) + row * p.y_stride + n;
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
            if (i < live) y[i * ys] = __float2bfloat16_rn(r[i]);
    }
}

template <int N, int G>
__global__ void __launch_bounds__(T_THREADS, 2) w4_tc_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const W4Params p) {
    using L = TcLayout<N>;
    constexpr int SB = T_UNIT / G;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto bar = [&](int i) { return base + L::BARS + 8u * i; };
    const uint32_t tmem_slot = base + L::BARS + 8u * L::N_BARS;

    const int ranks = p.ranks, rank = ranks > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int n0 = blockIdx.x / ranks * T_TILE, row0 = blockIdx.y * N;
    // Units go in pairs, a stage of codes each; what lies behind the last input is read as zeros and scaled by 0.
    const int pairs_all = (p.k + 2 * T_UNIT - 1) / (2 * T_UNIT);
    const int q_first = pairs_all * rank / ranks, pairs = pairs_all * (rank + 1) / ranks - q_first;
    const int units = 2 * pairs, groups = units * SB, g_first = q_first * (2 * SB);

    if (threadIdx.x == 0) {
        for (int i = 0; i < T_WSTAGES; ++i) {
            mbar_init(bar(L::W_FULL + i), 1);
            mbar_init(bar(L::W_EMPTY + i), 8);  // two units, four warps each
        }
        for (int i = 0; i < T_XSTAGES; ++i) mbar_init(bar(L::U_FULL + i), 5);  // both operands of a unit: four warps, and x
        for (int i = 0; i < T_RING; ++i) {
            mbar_init(bar(L::D_FULL + i), 1);
            mbar_init(bar(L::D_EMPTY + i), 4);
            mbar_init(bar(L::U_DONE + i), 1);
        }
        mbar_init(bar(L::DRAIN), 2);
        fence_mbar_init();
    }
    if (warp == 12) {
        tmem_alloc(tmem_slot, T_TMEM);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot));
    const uint32_t d0 = tmem + 2 * T_ACOLS;
    // Where a unit is one group its completion is the group's: one barrier tells both.  A warp that takes every other unit looks at every phase of
    // the barriers it looks at, because the rings' lengths are even, and none completes a second time before the warp has gone on.
    constexpr int DONE = SB == 1 ? L::D_FULL : L::U_DONE;

    auto unit_done = [&](int u) { return warp_wait(bar(DONE + (u & (T_RING - 1))), (u / T_RING) & 1, p.status); };

    if (warp < 8) {  // ---------------- codes to operands
        set_registers<T_REGS_WIDEN>(false);
        const int quarter = warp & 3, half = warp >> 2;
        const uint32_t row = base + (quarter * 32 + lane) * 128;
        const uint32_t a = tmem + (static_cast<uint32_t>(quarter) << 21) + half * T_ACOLS;  // tensor-memory lanes 32 quarter ..
        Ring<T_WSTAGES> w;
        for (int u = half; u < units; u += 2, w.next()) {
            if (u >= 2 && !unit_done(u - 2)) break;
            if (!warp_wait(bar(L::W_FULL + w.at), w.phase, p.status)) break;
            tc_fence_after();
            const uint32_t src = row + w.at * T_WBYTES;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 q = lds128(src + ((half * 4 + i) ^ (lane & 7)) * 16);
                uint32_t r[16];
                widen(q.x, r);
                widen(q.y, r + 4);
                widen(q.z, r + 8);
                widen(q.w, r + 12);
                tmem_st16(a + 16 * i, r);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bar(L::U_FULL + (u & (T_XSTAGES - 1))));
                mbar_arrive(bar(L::W_EMPTY + w.at));
            }
        }
    } else if (warp < 12) {  // ---------------- sums
        set_registers<T_REGS_SUM>(true);
        const int quarter = warp - 8, n = n0 + quarter * 32 + lane;
        const uint16_t* sc = p.scales + min(n, p.n - 1);
        const uint32_t d_lane = d0 + (static_cast<uint32_t>(quarter) << 21);
        // scales are fetched AHEAD groups early; the bits are converted where they are used, because a conversion waits for the load
        constexpr int AHEAD = 4;
        uint32_t s[AHEAD];
        int g_next = g_first;  // the group whose scale is fetched next
        sc += static_cast<size_t>(g_first) * p.n;
        auto fetch = [&](uint32_t& to) {
            // (16 bits into a 32-bit register: nothing here waits for them)
            asm volatile("{\n.reg .pred in;\nsetp.ne.u32 in, %2, 0;\nmov.u32 %0, 0;\n@in ld.global.nc.u16 %0, [%1];\n}\n"
                         : "=r"(to) : "l"(sc), "r"(g_next < p.groups ? 1 : 0));
            ++g_next;
            sc += p.n;
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (i < groups) fetch(s[i]);
        float acc[N];
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = 0.f;
        bool ok = true;
        for (int g0 = 0; ok && g0 < groups; g0 += AHEAD) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int g = g0 + i, d = i % T_DBUFS;
                if (g >= groups) break;
                if (!warp_wait(bar(L::D_FULL + (g & (T_RING - 1))), (g / T_RING) & 1, p.status)) { ok = false; break; }
                tc_fence_after();
                const float f = bf16_bits_to_float(s[i]);
                if (g + AHEAD < groups) fetch(s[i]);
#pragma unroll
                for (int c = 0; c < N / 16; ++c) {
                    uint32_t r[16];
                    tmem_ld16(d_lane + d * N + 16 * c, r);
                    tmem_ld_wait();
                    if (c == N / 16 - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(L::D_EMPTY + (g & (T_RING - 1))));
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[16 * c + e] = fmaf(__uint_as_float(r[e]), f, acc[16 * c + e]);
                }
            }
        }
        if (ranks == 1) {
#pragma unroll
            for (int r = 0; r < N; r += 16) tc_store_y<16>(p, row0 + r, n, false, acc + r, n < p.n ? p.rows - row0 - r : 0);
        } else {
            // the slices' sums side by side in each CTA's shared memory: the stages of codes are idle once the last product is complete and every
            // copy has landed
            float* mine = reinterpret_cast<float*>(smem);
            asm volatile("bar.sync 1, 160;" ::: "memory");  // with the warp that loads codes
#pragma unroll
            for (int r = 0; r < N; ++r) mine[r * T_TILE + quarter * 32 + lane] = acc[r];
        }
    } else {
        set_registers<T_REGS_REST>(false);
        const uint32_t leader = elect_one();
        if (warp == 12 || warp == 15) {  // ---------------- products: one warp the even units, one the odd
            constexpr uint32_t idesc = umma_idesc_bf16(T_TILE, N);
            const int odd = warp == 15 ? 1 : 0;
            uint32_t phase = 0;  // of the ring, at unit u
            bool ok = true;
            for (int u = odd; ok && u < units; u += 2) {
                const int at = u & (T_XSTAGES - 1);
                if (!warp_wait(bar(L::U_FULL + at), phase, p.status)) break;
                const uint64_t xd = umma_desc_k_sw128(base + L::X0 + at * L::XBYTES);
                const uint32_t a = tmem + odd * T_ACOLS;
#pragma unroll
                for (int b = 0; b < SB; ++b) {
                    // group g has accumulator g & 1, its use number g / 2; the use before has been read out
                    const int g = u * SB + b;
                    if (g >= T_DBUFS && !warp_wait(bar(L::D_EMPTY + ((g - T_DBUFS) & (T_RING - 1))), ((g - T_DBUFS) / T_RING) & 1, p.status)) { ok = false; break; }
                    tc_fence_after();
#pragma unroll
                    for (int i = 0; i < G / 16; ++i) {
                        const int k = b * (G / 16) + i;  // step of 16 inputs within the unit
                        mma_ts(leader, d0 + (g & 1) * N, a + k * 8, xd + static_cast<uint64_t>((k / 4) * (L::XHALF >> 4) + 2 * (k % 4)), idesc, i != 0 ? 1u : 0u);
                    }
                    mma_commit(leader, bar(L::D_FULL + (g & (T_RING - 1))));
                }
                if (SB > 1 && ok) mma_commit(leader, bar(L::U_DONE + (u & (T_RING - 1))));
                if (at >= 2) phase ^= 1u;
            }
            mma_commit(leader, bar(L::DRAIN));  // all that was issued completes before the CTA ends, also when a wait gave up
            warp_wait(bar(L::DRAIN), 0, p.status);
        } else if (warp == 13) {  // ---------------- x
            if (leader) tma_prefetch_desc(&map_x);
            int u = 0;
            Ring<T_XSTAGES> x;
            for (; u < units; ++u, x.next()) {
                if (u >= T_XSTAGES && !unit_done(u - T_XSTAGES)) break;
                if (leader) {
                    const int k = q_first * (2 * T_UNIT) + u * T_UNIT;
                    mbar_arrive_expect_tx(bar(L::U_FULL + x.at), L::XBYTES);
                    tma_load_2d(base + L::X0 + x.at * L::XBYTES, &map_x, k, row0, bar(L::U_FULL + x.at));
                    tma_load_2d(base + L::X0 + x.at * L::XBYTES + L::XHALF, &map_x, k + 64, row0, bar(L::U_FULL + x.at));
                }
                __syncwarp();
            }
            // copies that are under way land before the CTA ends
            for (int j = max(0, u - T_XSTAGES); j < u; ++j) warp_wait(bar(L::U_FULL + j % T_XSTAGES), (j / T_XSTAGES) & 1, p.status);
        } else if (warp == 14) {  // ---------------- codes
            if (leader) tma_prefetch_desc(&map_w);
            int j = 0;
            Ring<T_WSTAGES> w;
            for (; j < pairs; ++j, w.next()) {
                if (j >= T_WSTAGES && !warp_wait(bar(L::W_EMPTY + w.at), w.phase ^ 1u, p.status)) break;
                if (leader) {
                    mbar_arrive_expect_tx(bar(L::W_FULL + w.at), T_WBYTES);
                    tma_load_2d(base + w.at * T_WBYTES, &map_w, (q_first + j) * (T_UNIT / 2), n0, bar(L::W_FULL + w.at));
                }
                __syncwarp();
            }
            for (int i = max(0, j - T_WSTAGES); i < j; ++i) warp_wait(bar(L::W_FULL + i % T_WSTAGES), (i / T_WSTAGES) & 1, p.status);
            if (ranks > 1) asm volatile("bar.sync 1, 160;" ::: "memory");
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 12) tmem_dealloc(tmem, T_TMEM);
    if (ranks == 1) return;
    // rows dealt over the cluster
    cluster_arrive();
    cluster_wait();
    const int mine = (min(p.rows - row0, N) - rank + ranks - 1) / ranks;  // rows of this CTA: rank, rank + ranks, ..
    for (int i = threadIdx.x; i < mine * (T_TILE / 4); i += T_THREADS) {
        const int r = rank + ranks * (i / (T_TILE / 4)), c = i % (T_TILE / 4) * 4;
        float v[4] = {};
#pragma unroll 2
        for (int q = 0; q < ranks; ++q) {
            float f[4];
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]) : "r"(map_to_cta(base + 4u * (r * T_TILE + c), q)) : "memory");
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += f[e];
        }
        tc_store_y<4>(p, row0 + r, n0 + c, true, v, p.n - n0 - c);
    }
    __syncwarp();  // (whole warps arrive)
    cluster_arrive();  // no CTA leaves while another still reads its sums
    cluster_wait();
}

template <int N, int G>
cudaError_t launch_tc(const W4Params& p, const CUtensorMap& mw, const CUtensorMap& mx, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((p.n + T_TILE - 1) / T_TILE) * p.ranks, static_cast<unsigned>((p.rows + N - 1) / N));
    cfg.blockDim = dim3(T_THREADS);
    cfg.dynamicSmemBytes = TcLayout<N>::BYTES;
    cfg.stream = stream;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = p.ranks;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = p.ranks > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, w4_tc_kernel<N, G>, mw, mx, p);
}
template <int N>
cudaError_t launch_tc_group(const W4Params& p, const CUtensorMap& mw, const CUtensorMap& mx, cudaStream_t stream) {
    switch (p.group) {
        case 32: return launch_tc<N, 32>(p, mw, mx, stream);
        case 64: return launch_tc<N, 64>(p, mw, mx, stream);
        default: return launch_tc<N, 128>(p, mw, mx, stream);
    }
}

template <int N, int G>
cudaError_t tc_init_one() {
    cudaFuncAttributes a;
    cudaError_t e = cudaFuncGetAttributes(&a, w4_tc_kernel<N, G>);
    if (e != cudaSuccess) return e;
    // the split of the registers among the warp groups draws on what a CTA is launched with
    if (a.numRegs * T_THREADS < 32 * (8 * T_REGS_WIDEN + 4 * T_REGS_SUM + 4 * T_REGS_REST)) return cudaErrorInvalidKernelImage;
    return cudaFuncSetAttribute(w4_tc_kernel<N, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcLayout<N>::BYTES);
}
template <int N>
cudaError_t tc_init_group() {
    cudaError_t e = tc_init_one<N, 32>();
    if (e == cudaSuccess) e = tc_init_one<N, 64>();
    if (e == cudaSuccess) e = tc_init_one<N, 128>();
    return e;
}

}  // namespace

cudaError_t launch_w4_tc(W4Params p, int num_sms, cudaStream_t stream) {
    const int box = p.rows <= 16 ? 16 : p.rows <= 32 ? 32 : 64;
    CUtensorMap mw, mx;
    // (codes as pairs of bytes: boxes of 64 pairs, 128 outputs)
    if (make_tmap_bf16_2d(&mw, p.codes, p.n, p.k / 4, p.k / 4, T_TILE) != 0 || make_tmap_bf16_2d(&mx, p.x, p.rows, p.k, p.x_stride, box) != 0) return cudaErrorInvalidValue;
    // slices of the inputs, at least 4 units each, while two CTAs per SM are not filled
    const long long tiles = static_cast<long long>((p.n + T_TILE - 1) / T_TILE) * ((p.rows + box - 1) / box);
    const int units = (p.k + T_UNIT - 1) / T_UNIT;
    p.ranks = 1;
    while (p.ranks < 8 && tiles * p.ranks * 2 <= 2LL * num_sms && units >= p.ranks * 8) p.ranks *= 2;  // (at least two pairs each)
    return box == 16 ? launch_tc_group<16>(p, mw, mx, stream) : box == 32 ? launch_tc_group<32>(p, mw, mx, stream) : launch_tc_group<64>(p, mw, mx, stream);
}

cudaError_t w4_tc_init() {
    cudaError_t e = tc_init_group<16>();
    if (e == cudaSuccess) e = tc_init_group<32>();
    if (e == cudaSuccess) e = tc_init_group<64>();
    return e;
}

}  // namespace vl
