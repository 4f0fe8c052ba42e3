// Writing new keys and values into a paged cache, quantising them on the way, and reading a range back.
//
// One (token, kv head) vector x of head_dim entries is quantised on its own: a = max(max |x_d|, 2^-110),
// scale = a / Q, code_d = round(x_d * (Q / a)) to the nearest code, ties to even, with Q the largest code (448 for
// e4m3, 127 for int8); all of it in fp32: the factor Q / a and the product are each rounded to 24 bits, then the product
// to the code.  The floor under a keeps Q / a finite.  A vector with an infinite or NaN entry gets the scale NaN and codes
// 0: it reads back as NaN throughout, and attention sees NaN exactly in the rows that may see the token.  Reading is
// code * scale in fp32, and that rounded to the output type.
//
// Both kernels move every byte once and are bound by HBM (by latency for a decode step's few rows).  head_dim / 16 lanes
// share a vector of keys and one of values, 16-byte loads and stores, the maximum by shuffles: a lane then finds the row's
// place once for 64 bytes.  (8 entries per lane spent the time on finding places: 55 us for 8 x 4096 rows.)
// Measured, e4m3, 8 kv heads of 128: 8 x 4096 rows written 38 us = 5.3 TB/s; 4 x 16384 rows read back as bf16 66 us = 5.1 TB/s.
#include <cuda_fp8.h>

#include "paged.cuh"

namespace vl {

namespace {

constexpr int KV_THREADS = 256;
constexpr int KV_CACHED_CU = 1024;  // sequences whose boundaries are searched in shared memory
constexpr float kMinAmax = 7.70371977754894e-34f;  // 2^-110

// The packed row's sequence: the last b with cu_rows[b] <= row.
__device__ __forceinline__ int seq_of_row(const int* cu, int batch, int row) {
    int lo = 0, hi = batch - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cu[mid] <= row) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Where a packed row lives.  kind: 0 = belongs to no sequence, 1 = its position does not exist, 2 = page / off valid.
struct RowPlace {
    int kind, page, off;
};
__device__ __forceinline__ RowPlace place_of_row(const PagedRowsDev& r, const PagedCacheDev& c, const int* cu, int row, int* status) {
    RowPlace p = {0, 0, 0};
    const int b = seq_of_row(cu, r.batch, row);
    const SeqView s = load_seq(r, c.page_shift, b, status);
    if (row < s.row0 || row >= s.row0 + s.n) return p;
    const int pos = s.len - s.n + (row - s.row0);
    p.kind = 1;
    if (pos < 0) return p;
    p.page = __ldg(r.page_table + static_cast<size_t>(b) * r.table_width + (pos >> c.page_shift));
    p.off = pos & ((1 << c.page_shift) - 1);
    if (static_cast<unsigned>(p.page) >= static_cast<unsigned>(c.n_pages)) raise_status(status, VERILLM_DEV_PAGE_RANGE);
    else p.kind = 2;
    return p;
}

__device__ __forceinline__ const int* cached_cu(const PagedRowsDev& r, int* sm) {
    if (r.batch > KV_CACHED_CU) return r.cu_rows;
    for (int i = threadIdx.x; i < r.batch; i += KV_THREADS) sm[i] = __ldg(r.cu_rows + i);
    __syncthreads();
    return sm;
}

template <int DTYPE>
__device__ __forceinline__ uint2 quantise8(const uint4& x, float inv) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t r[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float f[4] = {bf16_lo(w[2 * h]) * inv, bf16_hi(w[2 * h]) * inv, bf16_lo(w[2 * h + 1]) * inv, bf16_hi(w[2 * h + 1]) * inv};
        if (DTYPE == VERILLM_KV_E4M3) {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[0], f[1]), __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[2], f[3]), __NV_SATFINITE, __NV_E4M3);
            r[h] = lo | (hi << 16);
        } else {  // |f| is at most 127 and a rounding, which rounds to 127
            const int i0 = __float2int_rn(f[0]), i1 = __float2int_rn(f[1]), i2 = __float2int_rn(f[2]), i3 = __float2int_rn(f[3]);
            r[h] = __byte_perm(__byte_perm(i0, i1, 0x0040), __byte_perm(i2, i3, 0x0040), 0x5410);
        }
    }
    return make_uint2(r[0], r[1]);
}

// The vector's codes (this lane's 16) and its scale; called by whole warps.
template <int DH, int DTYPE>
__device__ __forceinline__ uint4 quantise_vector(const uint4 (&x)[2], float* scale) {
    constexpr int LANES = DH / 16;
    constexpr float Q = DTYPE == VERILLM_KV_E4M3 ? 448.f : 127.f;
    uint32_t bits = max(abs_max8(x[0]), abs_max8(x[1]));
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) bits = max(bits, __shfl_xor_sync(0xFFFFFFFFu, bits, o));
    const bool finite = bits < 0x7F80u;
    const float amax = fmaxf(bf16_bits_to_float(bits), kMinAmax);
    *scale = finite ? __fdiv_rn(amax, Q) : __int_as_float(0x7FC00000);
    if (!finite) return make_uint4(0u, 0u, 0u, 0u);
    const float inv = __fdiv_rn(Q, amax);
    const uint2 a = quantise8<DTYPE>(x[0], inv), b = quantise8<DTYPE>(x[1], inv);
    return make_uint4(a.x, a.y, b.x, b.y);
}

template <int DH, int DTYPE>
__global__ void __launch_bounds__(KV_THREADS)
kv_write_kernel(const PagedCacheDev c, const PagedRowsDev r, const __nv_bfloat16* __restrict__ k, const __nv_bfloat16* __restrict__ v,
                long long row_stride, int* status) {
    constexpr int LANES = DH / 16, VECS = KV_THREADS / LANES;
    __shared__ int sm_cu[KV_CACHED_CU];
    const int* cu = cached_cu(r, sm_cu);
    const int lane = threadIdx.x % LANES;
    const long long n_vec = static_cast<long long>(r.n_rows) * c.n_kv_heads;
    // the bound is the block's, so that whole warps reach the shuffles
    for (long long i0 = static_cast<long long>(blockIdx.x) * VECS; i0 < n_vec; i0 += static_cast<long long>(gridDim.x) * VECS) {
        const long long i = i0 + threadIdx.x / LANES;
        const bool in = i < n_vec;
        const int row = in ? static_cast<int>(i / c.n_kv_heads) : 0;
        const int head = in ? static_cast<int>(i - static_cast<long long>(row) * c.n_kv_heads) : 0;
        const long long src = row * row_stride + head * DH + lane * 16;
        const uint4 *pk = reinterpret_cast<const uint4*>(k + src), *pv = reinterpret_cast<const uint4*>(v + src);
        const uint4 xk[2] = {__ldg(pk), __ldg(pk + 1)}, xv[2] = {__ldg(pv), __ldg(pv + 1)};
        const RowPlace p = place_of_row(r, c, cu, row, status);
        const bool store = in && p.kind == 2;
        const size_t vec = ((static_cast<size_t>(p.page) * c.n_kv_heads + head) << c.page_shift) + p.off;
        if (DTYPE == VERILLM_KV_BF16) {
            if (store) {
                uint4 *dk = reinterpret_cast<uint4*>(c.k) + (vec * LANES + lane) * 2, *dv = reinterpret_cast<uint4*>(c.v) + (vec * LANES + lane) * 2;
                dk[0] = xk[0];
                dk[1] = xk[1];
                dv[0] = xv[0];
                dv[1] = xv[1];
            }
        } else {
            float ks, vs;
            const uint4 kc = quantise_vector<DH, DTYPE>(xk, &ks), vc = quantise_vector<DH, DTYPE>(xv, &vs);
            if (store) {
                reinterpret_cast<uint4*>(c.k)[vec * LANES + lane] = kc;
                reinterpret_cast<uint4*>(c.v)[vec * LANES + lane] = vc;
                if (lane == 0) {
                    c.k_scale[vec] = ks;
                    c.v_scale[vec] = vs;
                }
            }
        }
    }
}

// four stored codes -> float
template <int DTYPE>
__device__ __forceinline__ void decode4(uint32_t w, float* f) {
    if (DTYPE == VERILLM_KV_E4M3) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const __half2_raw x = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> (16 * h)), __NV_E4M3);
            const float2 y = __half22float2(__half2(x));
            f[2 * h] = y.x;
            f[2 * h + 1] = y.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = static_cast<float>(static_cast<int8_t>(w >> (8 * i)));
    }
}

// One lane's 16 bytes of a stored vector (8 bf16 or 16 codes), times the scale, into the output.
template <int DTYPE, bool F32>
__device__ __forceinline__ void read_piece(const uint4& x, float scale, void* out, bool wide) {
    constexpr int E = DTYPE == VERILLM_KV_BF16 ? 8 : 16;
    if (DTYPE == VERILLM_KV_BF16 && !F32) {
        *reinterpret_cast<uint4*>(out) = x;
        return;
    }
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float f[E];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (DTYPE == VERILLM_KV_BF16) {
            f[2 * i] = bf16_lo(w[i]);
            f[2 * i + 1] = bf16_hi(w[i]);
        } else {
            decode4<DTYPE>(w[i], f + 4 * i);
        }
    }
    if (DTYPE != VERILLM_KV_BF16) {
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] *= scale;
    }
    constexpr int WORDS = F32 ? E : E / 2;
    uint32_t y[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) y[i] = F32 ? __float_as_uint(f[i]) : pack_bf16(f[2 * i], f[(2 * i + 1) % E]);
    if (WORDS >= 8 && wide) {  // whole sectors
#pragma unroll
        for (int i = 0; i < WORDS / 8; ++i)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(static_cast<char*>(out) + 32 * i), "r"(y[(8 * i) % WORDS]),
                         "r"(y[(8 * i + 1) % WORDS]), "r"(y[(8 * i + 2) % WORDS]), "r"(y[(8 * i + 3) % WORDS]), "r"(y[(8 * i + 4) % WORDS]),
                         "r"(y[(8 * i + 5) % WORDS]), "r"(y[(8 * i + 6) % WORDS]), "r"(y[(8 * i + 7) % WORDS])
                         : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) reinterpret_cast<uint4*>(out)[i] = make_uint4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
    }
}

template <int DH, int DTYPE, bool F32>
__global__ void __launch_bounds__(KV_THREADS)
kv_read_kernel(const PagedCacheDev c, const PagedRowsDev r, void* __restrict__ k, void* __restrict__ v, long long row_stride, bool wide, int* status) {
    constexpr int E = DTYPE == VERILLM_KV_BF16 ? 8 : 16, LANES = DH / E, VECS = KV_THREADS / LANES;
    __shared__ int sm_cu[KV_CACHED_CU];
    const int* cu = cached_cu(r, sm_cu);
    const int lane = threadIdx.x % LANES;
    // 16 rows of one head, then the next head: the rows of a page lie together in the pool
    const long long n_vec = static_cast<long long>((r.n_rows + 15) / 16) * 16 * c.n_kv_heads;
    for (long long i = static_cast<long long>(blockIdx.x) * VECS + threadIdx.x / LANES; i < n_vec; i += static_cast<long long>(gridDim.x) * VECS) {
        const long long q = i >> 4;
        const int block = static_cast<int>(q / c.n_kv_heads), head = static_cast<int>(q - static_cast<long long>(block) * c.n_kv_heads);
        const int row = block * 16 + static_cast<int>(i & 15);
        if (row >= r.n_rows) continue;
        const RowPlace p = place_of_row(r, c, cu, row, status);
        if (p.kind == 0) continue;  // behind the last sequence: left as it is
        const long long dst = (row * row_stride + head * DH + lane * E) * (F32 ? 4 : 2);
        uint4 xk = make_uint4(0u, 0u, 0u, 0u), xv = xk;
        float ks = 0.f, vs = 0.f;
        if (p.kind == 2) {
            const size_t vec = ((static_cast<size_t>(p.page) * c.n_kv_heads + head) << c.page_shift) + p.off;
            xk = __ldg(reinterpret_cast<const uint4*>(c.k) + vec * LANES + lane);
            xv = __ldg(reinterpret_cast<const uint4*>(c.v) + vec * LANES + lane);
            if (DTYPE != VERILLM_KV_BF16) {
                ks = __ldg(c.k_scale + vec);
                vs = __ldg(c.v_scale + vec);
            }
        }
        read_piece<DTYPE, F32>(xk, ks, static_cast<char*>(k) + dst, wide);
        read_piece<DTYPE, F32>(xv, vs, static_cast<char*>(v) + dst, wide);
    }
}

template <int DH, int DTYPE>
cudaError_t write_one(const PagedCacheDev& c, const PagedRowsDev& r, const void* k, const void* v, long long row_stride, int* status,
                      int num_sms, cudaStream_t stream) {
    constexpr int VECS = KV_THREADS / (DH / 16);
    const long long blocks = (static_cast<long long>(r.n_rows) * c.n_kv_heads + VECS - 1) / VECS;
    kv_write_kernel<DH, DTYPE><<<static_cast<unsigned>(blocks < 8LL * num_sms ? blocks : 8LL * num_sms), KV_THREADS, 0, stream>>>(
        c, r, reinterpret_cast<const __nv_bfloat16*>(k), reinterpret_cast<const __nv_bfloat16*>(v), row_stride, status);
    return cudaGetLastError();
}

template <int DH, int DTYPE, bool F32>
cudaError_t read_one(const PagedCacheDev& c, const PagedRowsDev& r, void* k, void* v, long long row_stride, int* status, int num_sms,
                     cudaStream_t stream) {
    constexpr int VECS = KV_THREADS / (DH / (DTYPE == VERILLM_KV_BF16 ? 8 : 16));
    const long long blocks = (static_cast<long long>((r.n_rows + 15) / 16) * 16 * c.n_kv_heads + VECS - 1) / VECS;
    // 32-byte stores where the rows allow them
    const bool wide = ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | static_cast<uintptr_t>(row_stride * (F32 ? 4 : 2))) & 31u) == 0;
    kv_read_kernel<DH, DTYPE, F32><<<static_cast<unsigned>(blocks < 8LL * num_sms ? blocks : 8LL * num_sms), KV_THREADS, 0, stream>>>(
        c, r, k, v, row_stride, wide, status);
    return cudaGetLastError();
}

template <int DH, int DTYPE>
cudaError_t read_as(const PagedCacheDev& c, const PagedRowsDev& r, void* k, void* v, long long row_stride, int out_f32, int* status,
                    int num_sms, cudaStream_t stream) {
    return out_f32 ? read_one<DH, DTYPE, true>(c, r, k, v, row_stride, status, num_sms, stream)
                   : read_one<DH, DTYPE, false>(c, r, k, v, row_stride, status, num_sms, stream);
}

}  // namespace

cudaError_t launch_kv_write(const PagedCacheDev& c, const PagedRowsDev& r, const void* k, const void* v, long long row_stride,
                            int* status, int num_sms, cudaStream_t stream) {
    const bool wide = c.head_dim == 128;
    switch (c.dtype) {
        case VERILLM_KV_BF16:
            return wide ? write_one<128, VERILLM_KV_BF16>(c, r, k, v, row_stride, status, num_sms, stream)
                        : write_one<64, VERILLM_KV_BF16>(c, r, k, v, row_stride, status, num_sms, stream);
        case VERILLM_KV_E4M3:
            return wide ? write_one<128, VERILLM_KV_E4M3>(c, r, k, v, row_stride, status, num_sms, stream)
                        : write_one<64, VERILLM_KV_E4M3>(c, r, k, v, row_stride, status, num_sms, stream);
        default:
            return wide ? write_one<128, VERILLM_KV_INT8>(c, r, k, v, row_stride, status, num_sms, stream)
                        : write_one<64, VERILLM_KV_INT8>(c, r, k, v, row_stride, status, num_sms, stream);
    }
}

cudaError_t launch_kv_read(const PagedCacheDev& c, const PagedRowsDev& r, void* k, void* v, long long row_stride, int out_f32,
                           int* status, int num_sms, cudaStream_t stream) {
    const bool wide = c.head_dim == 128;
    switch (c.dtype) {
        case VERILLM_KV_BF16:
            return wide ? read_as<128, VERILLM_KV_BF16>(c, r, k, v, row_stride, out_f32, status, num_sms, stream)
                        : read_as<64, VERILLM_KV_BF16>(c, r, k, v, row_stride, out_f32, status, num_sms, stream);
        case VERILLM_KV_E4M3:
            return wide ? read_as<128, VERILLM_KV_E4M3>(c, r, k, v, row_stride, out_f32, status, num_sms, stream)
                        : read_as<64, VERILLM_KV_E4M3>(c, r, k, v, row_stride, out_f32, status, num_sms, stream);
        default:
            return wide ? read_as<128, VERILLM_KV_INT8>(c, r, k, v, row_stride, out_f32, status, num_sms, stream)
                        : read_as<64, VERILLM_KV_INT8>(c, r, k, v, row_stride, out_f32, status, num_sms, stream);
    }
}

}  // namespace vl
