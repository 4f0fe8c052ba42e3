// Products with 4-bit weights: y[r][n] = sum_g s[g][n] * sum_{k in g} x[r][k] c[n][k] (+ residual[r][n]), codes c in -8 .. 7
// stored as c + 8, one bf16 scale per group of G = 32, 64 or 128 inputs; the quantisation that makes them, and its inverse.
//
// Arithmetic: a code is exact in bf16, so the tensor cores form the products x * c of a group exactly and add them in fp32; the
// group's sum is then multiplied by its scale and added to the running sum, both in fp32.  No weight is rounded again.
//
// w4_rows_kernel, up to 8 rows of x: bound by the weights' bytes.  A warp takes 16 outputs and all their inputs, or a part of them; weights stream from
// global memory straight into one operand of mma.sync, four chunks ahead, x is the other from shared memory, where the CTA laid it out in fragment
// order.  Warps are independent of one another until their sums meet.  The order of the inputs inside a product is free as long as both operands
// agree: a lane takes G / 4 consecutive ones, G / 8 bytes of codes.  A code becomes bf16 by its bits alone (0x4300 | u is 128 + u) and one exact
// subtraction of 136.
#include "common.cuh"
#include "kernels.h"

namespace vl {

namespace {

typedef __nv_bfloat16 bf16;

constexpr int W4_MAX_WARPS = 16;
constexpr int W4_MAX_SMEM = 224 * 1024;
constexpr int W4_CHUNK = 128;  // inputs per chunk

__device__ __forceinline__ void mma_bf16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same without an addend.
__device__ __forceinline__ void mma_bf16_16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// Codes i and i + 4 of a word as a pair of bf16.
__device__ __forceinline__ uint32_t code_pair(uint32_t q, int i) {
    uint32_t r;  // (the compiler makes two instructions of an and and an or with constants)
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(q >> (4 * i)), "r"(0x000F000Fu), "r"(0x43004300u));
    asm("sub.rn.bf16x2 %0, %0, %1;" : "+r"(r) : "r"(0x43084308u));
    return r;
}

// WORDS 32-bit words that are read once
template <int WORDS>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {
    if (WORDS == 4)
        asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1 % WORDS]), "=r"(w[2 % WORDS]), "=r"(w[3 % WORDS]) : "l"(p));
    else if (WORDS == 2)
        asm volatile("ld.global.nc.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1 % WORDS]) : "l"(p));
    else
        asm volatile("ld.global.nc.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
}
// The bits of a bf16 in a 32-bit register: nothing here waits for them.
__device__ __forceinline__ uint32_t load_bits16(const uint16_t* p) {
    uint32_t v;
    asm volatile("ld.global.nc.u16 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}

// One value of the result: the residual added, rounded to the output's type.
__device__ __forceinline__ void store_y(const W4Params& p, int row, int n, float v) {
    if (row >= p.rows || n >= p.n) return;
    if (p.residual) v += p.residual[row * p.res_stride + n];
    if (p.out_f32) reinterpret_cast<float*>(p.y)[row * p.y_stride + n] = v;
    else reinterpret_cast<bf16*>(p.y)[row * p.y_stride + n] = __float2bfloat16_rn(v);
}

// The codes of one chunk of a tile, outputs g and g + 8, and their scales.
template <int G>
struct Chunk {
    static constexpr int SB = W4_CHUNK / G, WORDS = G / 32;  // groups per chunk, words per lane and group
    uint32_t lo[4], hi[4], slo[SB], shi[SB];

    // code: this lane's bytes of the chunk's first group for output g, code_hi for output g + 8; scale, scale_hi likewise
    __device__ __forceinline__ void load(const W4Params& p, const uint8_t* code, const uint8_t* code_hi, const uint16_t* scale, const uint16_t* scale_hi, int group) {
#pragma unroll
        for (int b = 0; b < SB; ++b) {
            if (SB == 1 || group + b < p.groups) {
                load_words<WORDS>(code + b * (G / 2), lo + b * WORDS);
                load_words<WORDS>(code_hi + b * (G / 2), hi + b * WORDS);
                slo[b] = load_bits16(scale + static_cast<size_t>(b) * p.n);
                shi[b] = load_bits16(scale_hi + static_cast<size_t>(b) * p.n);
            } else {  // behind the last input: x is zero there
#pragma unroll
                for (int w = 0; w < WORDS; ++w) lo[b * WORDS + w] = hi[b * WORDS + w] = 0x88888888u;
                slo[b] = shi[b] = 0;
            }
        }
    }
    // acc += the chunk's products; x: the lane's fragments of the same inputs in shared memory, `words` apart
    __device__ __forceinline__ void multiply(uint32_t x, uint32_t words, float (&acc)[4]) const {
#pragma unroll
        for (int b = 0; b < SB; ++b) {
            float d[4];
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                const int k = b * WORDS + i;
                uint32_t f[4];
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(f[0]), "=r"(f[1]), "=r"(f[2]), "=r"(f[3]) : "r"(x + k * words));
                if (i == 0) mma_bf16_16816_first(d, code_pair(lo[k], 0), code_pair(hi[k], 0), code_pair(lo[k], 1), code_pair(hi[k], 1), f[0], f[1]);
                else mma_bf16_16816(d, code_pair(lo[k], 0), code_pair(hi[k], 0), code_pair(lo[k], 1), code_pair(hi[k], 1), f[0], f[1]);
                mma_bf16_16816(d, code_pair(lo[k], 2), code_pair(hi[k], 2), code_pair(lo[k], 3), code_pair(hi[k], 3), f[2], f[3]);
            }
            const float s0 = bf16_bits_to_float(slo[b]), s1 = bf16_bits_to_float(shi[b]);
            acc[0] = fmaf(d[0], s0, acc[0]);
            acc[1] = fmaf(d[1], s0, acc[1]);
            acc[2] = fmaf(d[2], s1, acc[2]);
            acc[3] = fmaf(d[3], s1, acc[3]);
        }
    }
};

// A warp takes every kw-th part of the inputs of one tile of 16 outputs; nothing but the final sum of its kw warps is shared.
template <int G>
__global__ void __launch_bounds__(W4_MAX_WARPS * 32) w4_rows_kernel(const W4Params p) {
    constexpr int SB = Chunk<G>::SB, WORDS = Chunk<G>::WORDS, AHEAD = 4;
    extern __shared__ __align__(16) uint8_t x_smem[];  // [chunk][word][row][t] pieces of 16 bytes; after them the warps' sums
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int kw = p.kw, sub = warp / kw, kidx = warp - sub * kw, tile = blockIdx.x * (blockDim.x / 32 / kw) + sub;
    const int chunks = (p.k + W4_CHUNK - 1) / W4_CHUNK;
    const int c0 = chunks * kidx / kw, c1 = tile < p.tiles ? chunks * (kidx + 1) / kw : c0;

    // (n is a multiple of 8: where a tile has 8 outputs only, they are computed twice)
    const int n0 = min(tile, p.tiles - 1) * 16 + g;
    const bool whole = n0 - g + 16 <= p.n;
    const uint8_t *code = p.codes + static_cast<size_t>(n0) * p.row_bytes + c0 * 64 + t * (G / 8), *code_hi = code + (whole ? 8 * static_cast<ptrdiff_t>(p.row_bytes) : 0);
    const uint16_t *scale = p.scales + static_cast<size_t>(c0) * SB * p.n + n0, *scale_hi = scale + (whole ? 8 : 0);
    const ptrdiff_t scale_step = static_cast<ptrdiff_t>(SB) * p.n;
    Chunk<G> w[AHEAD];
    auto load = [&](int i, int c) {  // the next chunk, number c, into stage i
        w[i].load(p, code, code_hi, scale, scale_hi, c * SB);
        code += 64;
        code_hi += 64;
        scale += scale_step;
        scale_hi += scale_step;
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (c0 + i < c1) load(i, c0 + i);

    // x in the order in which fragments are read, pairs (i, i + 4) like the codes'
    {
        constexpr int U = 4;  // loads in flight
        const unsigned per_row = chunks * 16, total = p.rows * per_row;
        for (unsigned i0 = threadIdx.x; i0 < total; i0 += U * blockDim.x) {
            uint4 v[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const unsigned i = i0 + j * blockDim.x, row = i / per_row, k8 = i - row * per_row;
                v[j] = make_uint4(0u, 0u, 0u, 0u);
                if (i < total && k8 * 8 < p.k) v[j] = __ldg(reinterpret_cast<const uint4*>(p.x + row * p.x_stride) + k8);
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const unsigned i = i0 + j * blockDim.x, row = i / per_row, k8 = i - row * per_row;
                if (i >= total) break;
                const int c = k8 >> 4, in = k8 & 15, b = in * 8 / G, rest = in - b * (G / 8);  // chunk, group within it, eighth of the group's inputs
                const int at = ((c * 4 + b * WORDS + rest % WORDS) * p.rows + row) * 4 + rest / WORDS;
                reinterpret_cast<uint4*>(x_smem)[at] = make_uint4(__byte_perm(v[j].x, v[j].z, 0x5410), __byte_perm(v[j].x, v[j].z, 0x7632),
                                                                  __byte_perm(v[j].y, v[j].w, 0x5410), __byte_perm(v[j].y, v[j].w, 0x7632));
            }
        }
    }
    __syncthreads();

    // (rows that do not exist are some other row again: their columns are not stored)
    const uint32_t words = p.rows * 64, per_chunk = 4 * words;
    uint32_t x = smem_u32(x_smem) + c0 * per_chunk + (min(g, p.rows - 1) * 4 + t) * 16;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int c = c0; c < c1; c += AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (c + i >= c1) break;
            w[i].multiply(x, words, acc);
            x += per_chunk;
            if (c + AHEAD + i < c1) load(i, c + AHEAD + i);
        }
    }
    float4 sum = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (kw > 1) {
        float4* part = reinterpret_cast<float4*>(x_smem + static_cast<size_t>(chunks) * per_chunk);
        part[warp * 32 + lane] = sum;
        __syncthreads();
        if (kidx != 0) return;
        for (int i = 1; i < kw; ++i) {  // in the order of the inputs
            const float4 v = part[(warp + i) * 32 + lane];
            sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
        }
    }
    if (tile >= p.tiles) return;
    store_y(p, 2 * t, n0, sum.x);
    store_y(p, 2 * t + 1, n0, sum.y);
    if (whole) {
        store_y(p, 2 * t, n0 + 8, sum.z);
        store_y(p, 2 * t + 1, n0 + 8, sum.w);
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

// Shared memory of the kernel for few rows: x, and the warps' sums.
size_t rows_smem(const W4Params& p, int warps) { return static_cast<size_t>((p.k + W4_CHUNK - 1) / W4_CHUNK) * W4_CHUNK * p.rows * 2 + warps * 512; }

template <int G>
cudaError_t launch_rows(W4Params& p, int num_sms, cudaStream_t stream) {
    // Small CTAs balance best as long as laying out x costs each little (4 warps, four CTAs per SM); with more of x one CTA of 16 warps per SM.
    // Measured, 8 rows x 28672 x 4096: 19 us with 16 warps, 41 with 4; one row x 57344 x 8192: 63 and 57.
    const bool small = rows_smem(p, 4) <= 20 * 1024;
    int warps = small ? 4 : 16;
    // A tile's inputs are divided among kw of a CTA's warps while all CTAs run at once and a warp keeps four chunks (eight ways: half as many
    // CTAs per SM, for long inputs only).  One row x 4096 x 14336: 10.6 us eight ways, 12.3 four, 34.8 undivided.
    const int chunks = (p.k + W4_CHUNK - 1) / W4_CHUNK;
    auto ctas = [&](int kw, int w) { return (p.tiles + w / kw - 1) / (w / kw); };
    p.kw = 1;
    while (p.kw < 8) {
        const int kw = 2 * p.kw, w = kw > warps ? kw : warps;
        if (chunks < (small && kw == 8 ? 64 : 4 * kw) || ctas(kw, w) > num_sms * (16 / w)) break;
        p.kw = kw;
        warps = w;
    }
    w4_rows_kernel<G><<<ctas(p.kw, warps), warps * 32, rows_smem(p, warps), stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t w4_init() {
    cudaError_t e = cudaFuncSetAttribute(w4_rows_kernel<32>, cudaFuncAttributeMaxDynamicSharedMemorySize, W4_MAX_SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(w4_rows_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, W4_MAX_SMEM);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(w4_rows_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, W4_MAX_SMEM);
    if (e == cudaSuccess) e = w4_tc_init();
    return e;
}

cudaError_t launch_w4_matvec(W4Params p, int num_sms, cudaStream_t stream) {
    p.groups = p.k / p.group;
    p.row_bytes = p.k / 2;
    p.tiles = (p.n + 15) / 16;
    if (p.rows > kW4FewRows || rows_smem(p, W4_MAX_WARPS) > W4_MAX_SMEM) return launch_w4_tc(p, num_sms, stream);
    switch (p.group) {
        case 32: return launch_rows<32>(p, num_sms, stream);
        case 64: return launch_rows<64>(p, num_sms, stream);
        default: return launch_rows<128>(p, num_sms, stream);
    }
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
