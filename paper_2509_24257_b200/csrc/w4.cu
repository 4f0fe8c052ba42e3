// Products with 4-bit weights: y[r][n] = sum_g s[g][n] * sum_{k in g} x[r][k] c[n][k] (+ residual[r][n]), codes c in -8 .. 7
// stored as c + 8, one bf16 scale per group of G = 32, 64 or 128 inputs; the quantisation that makes them, and its inverse.
//
// Arithmetic: a code is exact in bf16, so the tensor cores form the products x * c of a group exactly and add them in fp32; the
// group's sum is then multiplied by its scale and added to the running sum, both in fp32.  No weight is rounded again.
//
// w4_rows_kernel, up to 8 rows of x: bound by the weights' bytes.  A tile is 16 outputs; a warp takes CH chunks of 128 inputs of
// it and always the same chunks, so that its part of x stays in registers as operand fragments while weights stream from
// global memory straight into the other operand (the next tile's are requested before this one's are used).  The order of the inputs inside a
// product is free as long as both operands agree: a lane takes G / 4 consecutive ones, G / 8 bytes of codes.  A code becomes
// bf16 by its bits alone (0x4300 | u is 128 + u) and one exact subtraction of 136.  Long inputs are divided over a cluster, whose CTAs leave
// their sums of a tile in the shared memory of the tile's owner; sums are formed in a fixed order.
#include "common.cuh"
#include "kernels.h"

namespace vl {

namespace {

typedef __nv_bfloat16 bf16;

constexpr int W4_WARPS = 16;
constexpr int W4_THREADS = W4_WARPS * 32;
constexpr int W4_CHUNK = 128;  // inputs per chunk

__device__ __forceinline__ void mma_bf16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}

// Codes i and i + 4 of a word as a pair of bf16.
__device__ __forceinline__ uint32_t code_pair(uint32_t q, int i) {
    return sub_bf16x2(((q >> (4 * i)) & 0x000F000Fu) | 0x43004300u, 0x43084308u);
}

// WORDS 32-bit words that are read once
template <int WORDS>
__device__ __forceinline__ void load_words(const void* p, uint32_t* w) {
    if (WORDS == 4)
        asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1 % WORDS]), "=r"(w[2 % WORDS]), "=r"(w[3 % WORDS]) : "l"(p));
    else if (WORDS == 2)
        asm volatile("ld.global.nc.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1 % WORDS]) : "l"(p));
    else
        asm volatile("ld.global.nc.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
}

// A warp's share of one tile: codes of rows g and g + 8 and their scales.
template <int CH, int G>
struct TileRegs {
    static constexpr int SB = W4_CHUNK / G, WORDS = G / 32;  // groups per chunk, words per lane and group
    uint32_t lo[CH][4], hi[CH][4];
    uint16_t slo[CH][SB], shi[CH][SB];

    __device__ __forceinline__ void load(const W4Params& p, int tile, int chunk0, int lane) {
        const int g = lane >> 2, t = lane & 3;
        const int n0 = min(tile * 16 + g, p.n - 1), n1 = min(tile * 16 + g + 8, p.n - 1);  // rows behind the last are computed and not stored
        const uint8_t* base = p.codes + t * (G / 8);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int b = 0; b < SB; ++b) {
                const int group = (chunk0 + c) * SB + b;
                const bool in = group < p.groups;
                if (in) {
                    const size_t at = static_cast<size_t>(group) * (G / 2);
                    load_words<WORDS>(base + static_cast<size_t>(n0) * p.row_bytes + at, lo[c] + b * WORDS);
                    load_words<WORDS>(base + static_cast<size_t>(n1) * p.row_bytes + at, hi[c] + b * WORDS);
                    slo[c][b] = __ldg(p.scales + static_cast<size_t>(group) * p.n + n0);
                    shi[c][b] = __ldg(p.scales + static_cast<size_t>(group) * p.n + n1);
                } else {
#pragma unroll
                    for (int w = 0; w < WORDS; ++w) lo[c][b * WORDS + w] = hi[c][b * WORDS + w] = 0x88888888u;
                    slo[c][b] = shi[c][b] = 0;
                }
            }
        }
    }
};

// acc += the share's products; x: operand fragments of the same inputs.
template <int CH, int G>
__device__ __forceinline__ void multiply(const TileRegs<CH, G>& w, const uint32_t (&x)[CH][4][4], float (&acc)[4]) {
    constexpr int SB = TileRegs<CH, G>::SB, WORDS = TileRegs<CH, G>::WORDS;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int b = 0; b < SB; ++b) {
            float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                const int k = b * WORDS + i;
                const uint32_t lo = w.lo[c][k], hi = w.hi[c][k];
                mma_bf16_16816(d, code_pair(lo, 0), code_pair(hi, 0), code_pair(lo, 1), code_pair(hi, 1), x[c][k][0], x[c][k][1]);
                mma_bf16_16816(d, code_pair(lo, 2), code_pair(hi, 2), code_pair(lo, 3), code_pair(hi, 3), x[c][k][2], x[c][k][3]);
            }
            const float s0 = bf16_bits_to_float(w.slo[c][b]), s1 = bf16_bits_to_float(w.shi[c][b]);
            acc[0] = fmaf(d[0], s0, acc[0]);
            acc[1] = fmaf(d[1], s0, acc[1]);
            acc[2] = fmaf(d[2], s1, acc[2]);
            acc[3] = fmaf(d[3], s1, acc[3]);
        }
    }
}

// One value of the result: the residual added, rounded to the output's type.
__device__ __forceinline__ void store_y(const W4Params& p, int row, int n, float v) {
    if (row >= p.rows || n >= p.n) return;
    if (p.residual) v += p.residual[row * p.res_stride + n];
    if (p.out_f32) reinterpret_cast<float*>(p.y)[row * p.y_stride + n] = v;
    else reinterpret_cast<bf16*>(p.y)[row * p.y_stride + n] = __float2bfloat16_rn(v);
}

__device__ __forceinline__ void store_cluster(uint32_t addr, const float4& v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity, int* status) {
    const long long t0 = clock64();
    while (true) {
        uint32_t ok;
        asm volatile(
            "{\n"
            ".reg .pred p;\n"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n"
            "selp.u32 %0, 1, 0, p;\n"
            "}\n"
            : "=r"(ok)
            : "r"(bar), "r"(parity), "r"(kWaitSuspendNs)
            : "memory");
        if (ok) return true;
        if (clock64() - t0 > kWaitLimitCycles) {
            if (status) atomicCAS(status, 0, VERILLM_DEV_WAIT_TIMEOUT);
            return false;
        }
    }
}

// KW warps share a tile's inputs; the CTA's W4_WARPS / KW groups of warps take neighbouring tiles.  Clusters (of `ranks` CTAs, KW =
// W4_WARPS) divide longer inputs.  All warps of a cluster make the same number of steps.
template <int CH, int G>
__global__ void __launch_bounds__(W4_THREADS) w4_rows_kernel(const W4Params p) {
    __shared__ float4 part[2][W4_WARPS][32];
    __shared__ float4 joined[2][8][32];  // [slot][rank][lane] of the tiles that this CTA owns
    __shared__ uint64_t bars[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int kw = p.kw, sub = warp / kw, kidx = warp - sub * kw, per_step = W4_WARPS / kw;
    const int ranks = p.ranks, rank = ranks > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const int cluster = blockIdx.x / ranks, n_clusters = gridDim.x / ranks;
    const int chunk0 = (rank * kw + kidx) * CH;
    const int row0 = blockIdx.y * 8;

    TileRegs<CH, G> a, b;
    int step = cluster;
    a.load(p, min(step * per_step + sub, p.tiles - 1), chunk0, lane);

    // this lane's operand fragments of x: row row0 + g, inputs of its words; pairs (i, i + 4) like the codes'
    uint32_t x[CH][4][4];
    constexpr int SB = W4_CHUNK / G, WORDS = G / 32;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int group = (chunk0 + c) * SB + k / WORDS;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (row0 + g < p.rows && group < p.groups)
                v = __ldg(reinterpret_cast<const uint4*>(p.x + (row0 + g) * p.x_stride + static_cast<size_t>(group) * G + t * (G / 4) + (k % WORDS) * 8));
            x[c][k][0] = __byte_perm(v.x, v.z, 0x5410);
            x[c][k][1] = __byte_perm(v.x, v.z, 0x7632);
            x[c][k][2] = __byte_perm(v.y, v.w, 0x5410);
            x[c][k][3] = __byte_perm(v.y, v.w, 0x7632);
        }
    }
    if (ranks > 1) {
        if (threadIdx.x == 0) {
            mbar_init(smem_u32(&bars[0]), ranks);
            mbar_init(smem_u32(&bars[1]), ranks);
            fence_mbar_init();
        }
        cluster_arrive();
        cluster_wait();
    }

    int it = 0, owned = 0;
    auto one = [&](TileRegs<CH, G>& now, TileRegs<CH, G>& next) {
        const int tile = step * per_step + sub;
        step += n_clusters;
        if (step * per_step < p.tiles) next.load(p, min(step * per_step + sub, p.tiles - 1), chunk0, lane);
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        multiply<CH, G>(now, x, acc);
        float4 sum = make_float4(acc[0], acc[1], acc[2], acc[3]);
        const int buf = it & 1;
        if (kw > 1) {
            part[buf][warp][lane] = sum;
            __syncthreads();
        }
        // one warp of each tile adds the shares in order; the others go on (the buffer is written again two steps later, behind a
        // barrier that this warp has to reach first)
        if (kidx == it % kw) {
            if (kw > 1) {
                sum = part[buf][sub * kw][lane];
                for (int w = 1; w < kw; ++w) {
                    const float4 v = part[buf][sub * kw + w][lane];
                    sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
                }
            }
            bool mine = true;
            if (ranks > 1) {
                // the tile's owner gathers the cluster's sums.  A CTA is less than `ranks` steps ahead of another, because it waits for
                // all of them at each tile that it owns, so two slots suffice.
                const int owner = it % ranks, slot = (it / ranks) & 1;
                store_cluster(map_to_cta(smem_u32(&joined[slot][rank][lane]), owner), sum);
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&bars[slot]), owner));
                mine = owner == rank;
                if (mine) {
                    wait_cluster(smem_u32(&bars[slot]), (owned >> 1) & 1, p.status);
                    sum = joined[slot][0][lane];
                    for (int r = 1; r < ranks; ++r) {
                        const float4 v = joined[slot][r][lane];
                        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
                    }
                }
            }
            if (mine && tile < p.tiles) {
                store_y(p, row0 + 2 * t, tile * 16 + g, sum.x);
                store_y(p, row0 + 2 * t + 1, tile * 16 + g, sum.y);
                store_y(p, row0 + 2 * t, tile * 16 + g + 8, sum.z);
                store_y(p, row0 + 2 * t + 1, tile * 16 + g + 8, sum.w);
            }
        }
        if (ranks > 1 && it % ranks == rank) ++owned;
        ++it;
    };
    while (step * per_step < p.tiles) {
        one(a, b);
        if (step * per_step >= p.tiles) break;
        one(b, a);
    }
    if (ranks > 1) {  // no CTA leaves while another may still write to its shared memory
        cluster_arrive();
        cluster_wait();
    }
}

// --------------------------------------------------------------------------- quantisation
// scale = bf16(max |w| / 7), code = round(w / scale) to nearest, ties to even, at most 7 in magnitude.  A group with an infinite or NaN weight
// gets the scale NaN and codes 0: it stands for NaN.  G / 8 lanes per group, 16-byte reads; run once per model.
template <int G>
__global__ void __launch_bounds__(256) w4_quantise_kernel(const bf16* __restrict__ w, long long w_stride, uint8_t* __restrict__ codes,
                                                          bf16* __restrict__ scales, int n, int groups) {
    constexpr int LANES = G / 8, PER = 256 / LANES;
    const int lane = threadIdx.x % LANES;
    const long long total = static_cast<long long>(n) * groups;
    for (long long i0 = static_cast<long long>(blockIdx.x) * PER; i0 < total; i0 += static_cast<long long>(gridDim.x) * PER) {
        const long long i = min(i0 + threadIdx.x / LANES, total - 1);  // whole warps reach the shuffles; the last group may be written twice
        const long long row = i / groups;
        const int group = static_cast<int>(i - row * groups);
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(w + row * w_stride + static_cast<long long>(group) * G) + lane);
        const uint32_t q[4] = {v.x, v.y, v.z, v.w};
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = max(top, max(q[j] & 0x7FFFu, (q[j] >> 16) & 0x7FFFu));
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        const bool finite = top < 0x7F80u;
        const bf16 scale = finite ? __float2bfloat16_rn(__fdiv_rn(bf16_bits_to_float(top), 7.f)) : __ushort_as_bfloat16(0x7FC0);
        const float s = __bfloat162float(scale);
        uint32_t packed = 0x88888888u;
        if (finite && s > 0.f) {
            packed = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float f = j & 1 ? bf16_hi(q[j / 2]) : bf16_lo(q[j / 2]);
                const int c = max(-7, min(7, __float2int_rn(__fdiv_rn(f, s))));
                packed |= static_cast<uint32_t>(c + 8) << (4 * j);
            }
        }
        reinterpret_cast<uint32_t*>(codes)[i * LANES + lane] = packed;
        if (lane == 0) scales[static_cast<size_t>(group) * n + row] = scale;
    }
}

// out[n][k] = code * scale, rounded once to the output's type; 8 weights per thread.
template <typename OUT>
__global__ void __launch_bounds__(256) w4_dequantise_kernel(const uint8_t* __restrict__ codes, const uint16_t* __restrict__ scales, OUT* __restrict__ out,
                                                            long long out_stride, int n, int k, int group) {
    const int per_row = k / 8;
    const long long total = static_cast<long long>(n) * per_row;
    for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<long long>(gridDim.x) * 256) {
        const long long row = i / per_row;
        const int at = static_cast<int>(i - row * per_row) * 8;
        const uint32_t q = __ldg(reinterpret_cast<const uint32_t*>(codes) + i);
        const float s = bf16_bits_to_float(__ldg(scales + static_cast<size_t>(at / group) * n + row));
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = static_cast<float>(static_cast<int>((q >> (4 * j)) & 15u) - 8) * s;
        OUT* o = out + row * out_stride + at;
        if (sizeof(OUT) == 2) {
            *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
        } else {
            reinterpret_cast<float4*>(o)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4*>(o)[1] = make_float4(f[4], f[5], f[6], f[7]);
        }
    }
}

template <int CH, int G>
cudaError_t launch_rows(W4Params& p, int num_sms, cudaStream_t stream) {
    const int per_step = W4_WARPS / p.kw;
    const int steps = (p.tiles + per_step - 1) / per_step;
    const int clusters = max(1, min(steps, num_sms / p.ranks));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(clusters * p.ranks, (p.rows + 7) / 8);
    cfg.blockDim = dim3(W4_THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = p.ranks;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at;
    cfg.numAttrs = p.ranks > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, w4_rows_kernel<CH, G>, p);
}

template <int CH>
cudaError_t launch_group(W4Params& p, int num_sms, cudaStream_t stream) {
    switch (p.group) {
        case 32: return launch_rows<CH, 32>(p, num_sms, stream);
        case 64: return launch_rows<CH, 64>(p, num_sms, stream);
        default: return launch_rows<CH, 128>(p, num_sms, stream);
    }
}

}  // namespace

cudaError_t launch_w4_matvec(W4Params p, int num_sms, cudaStream_t stream) {
    p.groups = p.k / p.group;
    p.row_bytes = p.k / 2;
    p.tiles = (p.n + 15) / 16;
    const int chunks = (p.k + W4_CHUNK - 1) / W4_CHUNK;
    // one chunk per warp while a CTA's warps suffice, two then, and a cluster for what is longer
    const int ch = chunks > W4_WARPS ? 2 : 1, warps = (chunks + ch - 1) / ch;
    p.kw = 1;
    while (p.kw < warps && p.kw < W4_WARPS) p.kw *= 2;
    p.ranks = 1;
    while (p.ranks * p.kw < warps) p.ranks *= 2;
    if (p.ranks > 8) return cudaErrorInvalidValue;
    return ch == 1 ? launch_group<1>(p, num_sms, stream) : launch_group<2>(p, num_sms, stream);
}

cudaError_t launch_w4_quantise(const void* w, long long w_stride, void* codes, void* scales, int n, int k, int group, int num_sms, cudaStream_t stream) {
    const long long per = 256 / (group / 8), blocks = (static_cast<long long>(n) * (k / group) + per - 1) / per;
    const unsigned grid = static_cast<unsigned>(blocks < 16LL * num_sms ? blocks : 16LL * num_sms);
    const bf16* src = reinterpret_cast<const bf16*>(w);
    uint8_t* c = reinterpret_cast<uint8_t*>(codes);
    bf16* s = reinterpret_cast<bf16*>(scales);
    switch (group) {
        case 32: w4_quantise_kernel<32><<<grid, 256, 0, stream>>>(src, w_stride, c, s, n, k / group); break;
        case 64: w4_quantise_kernel<64><<<grid, 256, 0, stream>>>(src, w_stride, c, s, n, k / group); break;
        default: w4_quantise_kernel<128><<<grid, 256, 0, stream>>>(src, w_stride, c, s, n, k / group); break;
    }
    return cudaGetLastError();
}

cudaError_t launch_w4_dequantise(const void* codes, const void* scales, void* out, long long out_stride, int out_f32, int n, int k, int group,
                                 int num_sms, cudaStream_t stream) {
    const long long blocks = (static_cast<long long>(n) * (k / 8) + 255) / 256;
    const unsigned grid = static_cast<unsigned>(blocks < 16LL * num_sms ? blocks : 16LL * num_sms);
    const uint8_t* c = reinterpret_cast<const uint8_t*>(codes);
    const uint16_t* s = reinterpret_cast<const uint16_t*>(scales);
    if (out_f32) w4_dequantise_kernel<float><<<grid, 256, 0, stream>>>(c, s, reinterpret_cast<float*>(out), out_stride, n, k, group);
    else w4_dequantise_kernel<bf16><<<grid, 256, 0, stream>>>(c, s, reinterpret_cast<bf16*>(out), out_stride, n, k, group);
    return cudaGetLastError();
}

}  // namespace vl
