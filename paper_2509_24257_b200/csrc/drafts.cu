// Checking drafted tokens against the target's distribution with given random numbers.
//
// Row i of a sequence holds the logits of what follows its input token i; p = softmax(l / T), q the draft's distribution of the same row (or
// one at the drafted token).  The token x of row i + 1 is accepted iff u q(x) < p(x).  The first that is not is replaced by a draw from
// max(0, p - q), after the last one a token is drawn from p, both as the first v whose running sum exceeds s times the total.
//
// What comes out are whole numbers, so the arithmetic has to be good to the border: a draw among 10^5 tokens lies within 10^-6 of one
// often enough.  Two kernels:
//
// draft_rows_kernel, bound by HBM: maximum and sum of exp2 in fp32 of every row that counts, divided over the vocabulary, one pass.
// draft_verify_kernel, a cluster per sequence: joins these, accepts what is clear at fp32's error, decides the rows next to the border from
// sums in 64 bits, and draws by sums in 64 bits: over CTAs, warps, steps of a warp, lanes and entries, at each level the last part that begins at or before
// the drawn point and is not empty.
#include "common.cuh"
#include "kernels.h"

namespace vl {

namespace {

typedef __nv_bfloat16 bf16;

constexpr int DR_THREADS = 256;
constexpr int DR_UNROLL = 4;       // 16-byte blocks in flight per thread
constexpr int DV_THREADS = 512;
constexpr int DV_WARPS = DV_THREADS / 32;
constexpr float kMinTemp = 7.8886090522101181e-31f, kMaxTemp = 1.2676506002282294e30f;  // 2^-100, 2^100
constexpr double kLog2e = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

template <typename T>
struct Row {
    static constexpr int E = 16 / sizeof(T);  // entries per block
    const T* base;
    int vocab, off, blocks;  // the row begins `off` entries into its first 16-byte block
    __device__ __forceinline__ Row(const void* p, long long stride, long long row, int v) {
        base = reinterpret_cast<const T*>(p) + row * stride;
        vocab = v;
        off = static_cast<int>((reinterpret_cast<uintptr_t>(base) & 15u) / sizeof(T));
        blocks = (v + off + E - 1) / E;
    }
    // Entries [j0, j0 + E), -inf outside the row.
    __device__ __forceinline__ void load(int j0, float (&f)[E]) const {
        if (j0 >= 0 && j0 + E <= vocab && (reinterpret_cast<uintptr_t>(base + j0) & 15u) == 0) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(base + j0));
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < E; ++i)
                f[i] = sizeof(T) == 4 ? __uint_as_float(w[i % 4]) : i & 1 ? bf16_hi(w[i / 2 % 4]) : bf16_lo(w[i / 2 % 4]);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) f[i] = j0 + i >= 0 && j0 + i < vocab ? entry(j0 + i) : -INFINITY;
        }
    }
    __device__ __forceinline__ float entry(int j) const {
        if (sizeof(T) == 4) return __ldg(reinterpret_cast<const float*>(base) + j);
        return bf16_bits_to_float(__ldg(reinterpret_cast<const unsigned short*>(base) + j));
    }
};

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ bool temp_valid(float t) { return t == 0.f || (t >= kMinTemp && t <= kMaxTemp); }
__device__ __forceinline__ float temp_of(const DraftParams& p, int b) { return p.temperature ? __ldg(p.temperature + b) : 1.f; }

__device__ __forceinline__ void raise(int* status, int code) {
    if (status) atomicCAS(status, 0, code);
}

struct SeqRows {
    int row0, n;
    bool bad;  // outside what the buffers hold
};
__device__ __forceinline__ SeqRows seq_rows(const DraftParams& p, int b) {
    const int c0 = __ldg(p.cu_rows + b), c1 = __ldg(p.cu_rows + b + 1);
    SeqRows s;
    s.row0 = min(max(c0, 0), p.n_rows);
    s.n = min(max(c1, s.row0), p.n_rows) - s.row0;
    s.bad = c0 < 0 || c1 < c0 || c1 > p.n_rows || s.n > p.max_rows;
    return s;
}

// Statistics of one part of a row: x = maximum, y = sum of exp2((l - maximum) log2e / T), NaN if an entry is NaN or +inf; z = index of the
// first maximum where T = 0.
template <typename T>
__global__ void __launch_bounds__(DR_THREADS) draft_rows_kernel(const DraftParams p) {
    constexpr int E = Row<T>::E;
    __shared__ int sm_seq;
    __shared__ float sm_m[DR_THREADS / 32], sm_s[DR_THREADS / 32];
    __shared__ int sm_i[DR_THREADS / 32];
    const int row = blockIdx.x, splits = gridDim.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool draft = blockIdx.z == 1;
    const Row<T> r(draft ? p.draft : p.target, draft ? p.draft_stride : p.target_stride, row, p.vocab);
    const int per = (r.blocks + splits - 1) / splits;
    const int b0 = blockIdx.y * per, b1 = min(b0 + per, r.blocks);

    // the first blocks are on their way while the row's sequence is looked up
    float f[DR_UNROLL][E];
    auto fetch = [&](int b) {
#pragma unroll
        for (int u = 0; u < DR_UNROLL; ++u) {
            if (b + u * DR_THREADS < b1) {
                r.load((b + u * DR_THREADS) * E - r.off, f[u]);
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) f[u][i] = -INFINITY;
            }
        }
    };
    fetch(b0 + tid);
    pdl_launch_dependents();
    if (tid == 0) sm_seq = -1;
    __syncthreads();
    for (int b = tid; b < p.batch; b += DR_THREADS) {
        const SeqRows s = seq_rows(p, b);
        if (!s.bad && row >= s.row0 && row < s.row0 + s.n && (!draft || row + 1 < s.row0 + s.n)) sm_seq = b;
    }
    __syncthreads();
    const int seq = sm_seq;
    if (seq < 0) return;  // no sequence's row, or a draft row that nothing follows
    const float temp = temp_of(p, seq);
    const bool greedy = temp == 0.f;
    if (!temp_valid(temp) || (greedy && draft)) return;
    const float c = greedy ? 0.f : static_cast<float>(kLog2e / static_cast<double>(temp));

    float m = -INFINITY, s = 0.f;
    int at = 0x7FFFFFFF;
    for (int b = b0 + tid; b < b1; b += DR_THREADS * DR_UNROLL) {
        if (b != b0 + tid) fetch(b);
        if (greedy) {
#pragma unroll
            for (int u = 0; u < DR_UNROLL; ++u)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float v = f[u][i];
                    if (v > m) {
                        m = v;
                        at = (b + u * DR_THREADS) * E - r.off + i;
                    }
                    if (v != v) s = v;
                }
            continue;
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < DR_UNROLL; ++u)
#pragma unroll
            for (int i = 0; i < E; ++i) top = fmaxf(top, f[u][i]);
        // an entry of -inf with nothing finite before it: any finite reference does
        const float ref = top == -INFINITY ? 0.f : top;
        float add[DR_UNROLL];
#pragma unroll
        for (int u = 0; u < DR_UNROLL; ++u) {
            add[u] = 0.f;
#pragma unroll
            for (int i = 0; i < E; ++i) add[u] += exp2_approx((f[u][i] - ref) * c);
        }
        s = m == -INFINITY ? s : s * exp2_approx((m - ref) * c);
#pragma unroll
        for (int u = 0; u < DR_UNROLL; ++u) s += add[u];
        m = top;
    }
    // join: (m, s) pairs by their larger maximum, in a fixed order
    auto join = [&](float om, float os, int oi) {
        const float top = fmaxf(m, om);
        if (greedy) {
            if (om > m || (om == m && oi < at)) at = oi;
            if (os != os) s = os;
        } else {
            const float a = m == top ? s : s * exp2_approx((m - top) * c), b = om == top ? os : os * exp2_approx((om - top) * c);
            s = a + b;
        }
        m = top;
    };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        join(__shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o), __shfl_xor_sync(0xFFFFFFFFu, at, o));
    if (lane == 0) {
        sm_m[warp] = m;
        sm_s[warp] = s;
        sm_i[warp] = at;
    }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < DR_THREADS / 32; ++w) join(sm_m[w], sm_s[w], sm_i[w]);
        p.stats[(static_cast<size_t>(draft ? p.n_rows : 0) + row) * splits + blockIdx.y] = make_float4(m, s, __int_as_float(at), 0.f);
    }
}

// exp(d / T) for d <= 0 in 64 bits: 2^(j/64) from a table and a polynomial of degree 4 for the rest, |r| <= ln 2 / 128 (a table-driven
// exponential after P. T. P. Tang, 1989), relative error below 1e-13.
struct Exp64 {
    const double* table;  // 2^(j / 64), shared memory
    double inv_t, scale;  // 1 / T, 64 / (T ln 2)
    float floor;          // d below this: 0
    __device__ __forceinline__ double operator()(float l, float top) const {
        const float df = l - top;
        if (!(df > floor)) return 0.0;
        const double d = static_cast<double>(l) - static_cast<double>(top);
        const double big = fma(d, scale, 6755399441055744.0);  // 1.5 2^52: the nearest integer in the low bits
        const int n = __double2loint(big);
        const double r = fma(big - 6755399441055744.0, -kLn2 / 64.0, d * inv_t);
        double e = fma(r, 1.0 / 24.0, 1.0 / 6.0);
        e = fma(r, e, 0.5);
        e = fma(r, e, 1.0);
        e = fma(r, e, 1.0);
        e *= table[n & 63];
        return __hiloint2double(__double2hiint(e) + ((n >> 6) << 20), __double2loint(e));
    }
};

// What the running sums are made of.
struct Weights {
    int kind;       // 0: p; 1: p without token x; 2: max(0, p - q)
    int x;
    float pm, qm;   // the rows' maxima
    double a, b;    // kind 2: a e_p - b e_q, a = sum e_q, b = sum e_p
};

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
__device__ __forceinline__ double load_cluster64(uint32_t addr) {
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
    return v;
}

template <typename T>
__device__ __forceinline__ void weights_of(const Row<T>& rp, const Row<T>& rq, const Exp64& ex, const Weights& w, int j0, double (&v)[Row<T>::E]) {
    constexpr int E = Row<T>::E;
    float f[E];
    rp.load(j0, f);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = ex(f[i], w.pm);
    if (w.kind == 1) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (j0 + i == w.x) v[i] = 0.0;
    } else if (w.kind == 2) {
        rq.load(j0, f);
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = fmax(0.0, __dsub_rn(__dmul_rn(w.a, v[i]), __dmul_rn(w.b, ex(f[i], w.qm))));  // (no fma: 0 where p = q)
    }
}

template <typename T>
__global__ void __launch_bounds__(DV_THREADS) draft_verify_kernel(const DraftParams p) {
    constexpr int E = Row<T>::E;
    __shared__ double table[64];
    __shared__ double warp_tot[2][DV_WARPS];
    __shared__ double cta_tot[4];  // two pairs, used in turn
    __shared__ float sm_pm[kDraftMaxRows], sm_ps[kDraftMaxRows], sm_qm[kDraftMaxRows];
    __shared__ int sm_code[kDraftMaxRows], sm_arg[kDraftMaxRows];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ranks = p.ranks, rank = ranks > 1 ? static_cast<int>(cluster_ctarank()) : 0, b = blockIdx.x / ranks;
    const SeqRows s = seq_rows(p, b);
    const float temp = temp_of(p, b);
    const bool greedy = temp == 0.f;
    if (tid < 64) table[tid] = exp2(tid / 64.0);
    pdl_wait();
    if (s.bad && tid == 0 && rank == 0) raise(p.status, VERILLM_DEV_ROWS_RANGE);
    if (s.bad || s.n == 0 || !temp_valid(temp)) {  // (the whole cluster)
        if (rank == 0) {
            for (int i = tid; i < s.n; i += DV_THREADS) {
                p.out_tokens[s.row0 + i] = -1;
                if (p.logp) p.logp[s.row0 + i] = 0.f;
            }
            if (tid == 0) {
                if (!s.bad && s.n > 0) raise(p.status, VERILLM_DEV_LOGITS);
                p.n_emitted[b] = 0;
                if (p.new_len) p.new_len[b] = p.kv_len[b] - (s.bad ? 0 : s.n);
            }
        }
        return;
    }
    const float c = greedy ? 0.f : static_cast<float>(kLog2e / static_cast<double>(temp));
    const double inv_t = greedy ? 1.0 : 1.0 / static_cast<double>(temp);
    Exp64 ex;
    ex.table = table;
    ex.inv_t = inv_t;
    ex.scale = inv_t * (64.0 / kLn2);
    ex.floor = fmaxf(-700.f * temp, -3.0e38f);

    // ---- every row: its statistics and what fp32 says of the token that follows it
    // 0 accepted, 1 rejected, 2 too near to say, 3 no distribution, 4 the last row
    for (int i = warp; i < s.n; i += DV_WARPS) {
        const int row = s.row0 + i;
        auto gather = [&](int which, float& m, float& sum, int& at) {
            m = -INFINITY;
            sum = 0.f;
            at = 0x7FFFFFFF;
            if (lane < p.splits) {
                const float4 v = __ldcg(p.stats + (static_cast<size_t>(which ? p.n_rows : 0) + row) * p.splits + lane);
                m = v.x;
                sum = v.y;
                at = __float_as_int(v.z);
            }
            const float top = warp_max(m);
            if (greedy) {
                at = m == top ? at : 0x7FFFFFFF;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) at = min(at, __shfl_xor_sync(0xFFFFFFFFu, at, o));
                sum = warp_sum(sum);  // only whether it is NaN
            } else {
                sum = warp_sum(m == -INFINITY ? sum : sum * exp2_approx((m - top) * c));
            }
            m = top;
        };
        float pm, ps, qm = 0.f, qs = 1.f;
        int arg, unused;
        gather(0, pm, ps, arg);
        bool valid = fabsf(pm) < INFINITY && ps == ps && (greedy || ps < INFINITY);
        int code = 4;
        const bool follows = i + 1 < s.n;
        if (follows) {
            const int x = __ldg(p.tokens + row + 1);
            const bool in = x >= 0 && x < p.vocab;
            if (!in && lane == 0 && rank == 0) raise(p.status, VERILLM_DEV_TOKEN_RANGE);
            if (greedy) {
                code = x == arg ? 0 : 1;
            } else {
                if (p.draft) {
                    gather(1, qm, qs, unused);
                    valid = valid && fabsf(qm) < INFINITY && qs == qs && qs < INFINITY;
                }
                code = 1;
                if (in) {
                    const Row<T> rp(p.target, p.target_stride, row, p.vocab);
                    const float dp = rp.entry(x) - pm, lp = dp > ex.floor ? dp * c - log2f(ps) : -INFINITY;
                    float lq = 0.f;
                    if (p.draft) {
                        const Row<T> rq(p.draft, p.draft_stride, row, p.vocab);
                        const float dq = rq.entry(x) - qm;
                        lq = dq > ex.floor ? dq * c - log2f(qs) : -INFINITY;
                    }
                    const float u = __ldg(p.accept_u + row + 1), lu = log2f(u);
                    // lp and lq are off by less than 2^-21 of what was added up in them and 2^-19 of 1 (sums of exp2.approx)
                    const float diff = lu + lq - lp, near = 1e-5f * (4.f + fabsf(lp) + log2f(ps) + (p.draft ? fabsf(lq) + log2f(qs) : 0.f) + fabsf(lu));
                    if (u != u) code = 1;
                    else if (diff < -near || (u <= 0.f && lp > -INFINITY)) code = 0;
                    else if (diff > near || lp == -INFINITY) code = 1;
                    else code = 2;
                    if (lq == -INFINITY && lp > -INFINITY && u == u) code = 0;  // u * 0 < p
                }
            }
        }
        if (!valid) code = 3;
        if (lane == 0) {
            sm_code[i] = code;
            sm_arg[i] = arg;
            sm_pm[i] = pm;
            sm_ps[i] = ps;
            sm_qm[i] = qm;
        }
    }
    __syncthreads();

    // ---- sums in 64 bits over the cluster
    const int blocks = (p.vocab + E - 1) / E + 1;  // of any row, whatever its alignment
    const int per_cta = (blocks + ranks - 1) / ranks, per_warp = (per_cta + DV_WARPS - 1) / DV_WARPS;
    const int wb0 = rank * per_cta + warp * per_warp;
    const int wb1 = min(min(wb0 + per_warp, (rank + 1) * per_cta), blocks);
    int turn = 0;
    // totals of two running sums over the cluster; before[k]: of the CTAs before this one
    auto cluster_totals = [&](double v0, double v1, double (&total)[2], double (&mine)[2]) {
        v0 = warp_sum64(v0);
        v1 = warp_sum64(v1);
        if (lane == 0) {
            warp_tot[0][warp] = v0;
            warp_tot[1][warp] = v1;
        }
        __syncthreads();
        mine[0] = mine[1] = 0.0;
        for (int w = 0; w < DV_WARPS; ++w) {
            mine[0] += warp_tot[0][w];
            mine[1] += warp_tot[1][w];
        }
        if (tid == 0) {
            cta_tot[2 * turn] = mine[0];
            cta_tot[2 * turn + 1] = mine[1];
        }
        if (ranks > 1) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
        total[0] = total[1] = 0.0;
        for (int r = 0; r < ranks; ++r) {
            total[0] += ranks > 1 ? load_cluster64(map_to_cta(smem_u32(&cta_tot[2 * turn]), r)) : cta_tot[2 * turn];
            total[1] += ranks > 1 ? load_cluster64(map_to_cta(smem_u32(&cta_tot[2 * turn + 1]), r)) : cta_tot[2 * turn + 1];
        }
        turn ^= 1;
    };
    auto row_sums = [&](int i, double (&total)[2]) {  // sums of e_p and e_q of row i
        const Row<T> rp(p.target, p.target_stride, s.row0 + i, p.vocab), rq(p.draft ? p.draft : p.target, p.draft ? p.draft_stride : p.target_stride, s.row0 + i, p.vocab);
        double sp = 0.0, sq = 0.0, mine[2];
        for (int k = wb0 + lane; k < wb1; k += 32) {
            float f[E];
            rp.load(k * E - rp.off, f);
#pragma unroll
            for (int e = 0; e < E; ++e) sp += ex(f[e], sm_pm[i]);
            if (p.draft) {
                rq.load(k * E - rp.off, f);
#pragma unroll
                for (int e = 0; e < E; ++e) sq += ex(f[e], sm_qm[i]);
            }
        }
        cluster_totals(sp, sq, total, mine);
    };

    // ---- how many are accepted
    int stop = 0, code = 4;
    double sums[2] = {0.0, 0.0};
    bool have_sums = false;
    for (; stop < s.n; ++stop) {
        code = sm_code[stop];
        have_sums = false;
        if (code == 2) {
            row_sums(stop, sums);
            have_sums = true;
            const int x = __ldg(p.tokens + s.row0 + stop + 1);
            const Row<T> rp(p.target, p.target_stride, s.row0 + stop, p.vocab);
            const double ep = ex(rp.entry(x), sm_pm[stop]), u = static_cast<double>(__ldg(p.accept_u + s.row0 + stop + 1));
            if (p.draft) {
                const Row<T> rq(p.draft, p.draft_stride, s.row0 + stop, p.vocab);
                code = u * ex(rq.entry(x), sm_qm[stop]) * sums[0] < ep * sums[1] ? 0 : 1;
            } else {
                code = u * sums[0] < ep ? 0 : 1;
            }
        }
        if (code != 0) break;
    }
    // (the last row's code is never 0: stop < n)

    if (rank == 0) {
        for (int i = tid; i < s.n; i += DV_THREADS) {
            const int row = s.row0 + i;
            int tok = -1;
            float lp = 0.f;
            if (i < stop) {
                tok = __ldg(p.tokens + row + 1);
                if (!greedy) {
                    const Row<T> rp(p.target, p.target_stride, row, p.vocab);
                    lp = static_cast<float>(kLn2) * ((rp.entry(tok) - sm_pm[i]) * c - log2f(sm_ps[i]));
                }
            } else if (i == stop) {
                if (code != 3 && !greedy) continue;  // written by whoever draws it
                if (code != 3) tok = sm_arg[i];
            }
            p.out_tokens[row] = tok;
            if (p.logp) p.logp[row] = lp;
        }
        if (tid == 0) {
            const int emitted = code == 3 ? stop : stop + 1;
            if (code == 3) raise(p.status, VERILLM_DEV_LOGITS);
            p.n_emitted[b] = emitted;
            if (p.new_len) p.new_len[b] = p.kv_len[b] - s.n + emitted;
        }
    }
    if (code == 3 || greedy) {
        if (ranks > 1) {  // another CTA may still read this one's sums
            cluster_arrive();
            cluster_wait();
        }
        return;
    }

    // ---- the draw
    const Row<T> rp(p.target, p.target_stride, s.row0 + stop, p.vocab), rq(p.draft ? p.draft : p.target, p.draft ? p.draft_stride : p.target_stride, s.row0 + stop, p.vocab);
    Weights w;
    w.pm = sm_pm[stop];
    w.qm = sm_qm[stop];
    w.kind = code == 4 ? 0 : p.draft ? 2 : 1;
    w.x = code == 4 ? -1 : __ldg(p.tokens + s.row0 + stop + 1);
    if (w.kind == 2) {
        if (!have_sums) row_sums(stop, sums);
        w.a = sums[1];
        w.b = sums[0];
    }
    double total[2], mine[2];
    while (true) {
        double v = 0.0;
        for (int k = wb0 + lane; k < wb1; k += 32) {
            double x[E];
            weights_of<T>(rp, rq, ex, w, k * E - rp.off, x);
#pragma unroll
            for (int e = 0; e < E; ++e) v += x[e];
        }
        cluster_totals(v, 0.0, total, mine);
        if (total[0] > 0.0 || w.kind == 0) break;
        w.kind = 0;  // p nowhere above q (they are the same and the number was 1): drawn from p
    }
    const double u = fmin(fmax(static_cast<double>(__ldg(p.sample_u + b)), 0.0), 1.0), point = u * total[0];
    // the last CTA that begins at or before the point and is not empty
    int owner = 0;
    double before = 0.0, base = 0.0;
    for (int r = 0; r < ranks; ++r) {
        const double v = ranks > 1 ? load_cluster64(map_to_cta(smem_u32(&cta_tot[2 * (turn ^ 1)]), r)) : cta_tot[2 * (turn ^ 1)];
        if (v > 0.0 && before <= point) {
            owner = r;
            base = before;
        }
        before += v;
    }
    if (owner == rank) {
        int ow = 0;
        double at = base, start = base;
        for (int k = 0; k < DV_WARPS; ++k) {
            const double v = warp_tot[0][k];
            if (v > 0.0 && at <= point) {
                ow = k;
                start = at;
            }
            at += v;
        }
        if (warp == ow) {
            int token = -1;
            double run = start;
            for (int k0 = wb0; k0 < wb1; k0 += 32) {
                const int k = k0 + lane;
                double x[E], sum = 0.0;
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = 0.0;
                if (k < wb1) weights_of<T>(rp, rq, ex, w, k * E - rp.off, x);
#pragma unroll
                for (int e = 0; e < E; ++e) sum += x[e];
                double incl = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                    if (lane >= o) incl += v;
                }
                const double begin = run + (incl - sum);
                const unsigned who = __ballot_sync(0xFFFFFFFFu, sum > 0.0 && begin <= point);
                if (who) {
                    int tok = -1;
                    double r = begin;
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        if (x[e] > 0.0 && r <= point) tok = k * E - rp.off + e;
                        r += x[e];
                    }
                    token = __shfl_sync(0xFFFFFFFFu, tok, 31 - __clz(who));
                }
                run += __shfl_sync(0xFFFFFFFFu, incl, 31);
            }
            if (lane == 0) {
                p.out_tokens[s.row0 + stop] = token;
                if (p.logp) p.logp[s.row0 + stop] = token < 0 ? 0.f : static_cast<float>(kLn2) * ((rp.entry(token) - w.pm) * c - log2f(sm_ps[stop]));
            }
        }
    }
    if (ranks > 1) {
        cluster_arrive();
        cluster_wait();
    }
}

}  // namespace

// Parts that a row is divided into: 16384 entries each where that gives every SM four, down to 1024 where it does not; a lane joins each.
static int draft_splits(int n_rows, int vocab, int num_sms) {
    int per = 16384;
    while (per > 1024 && (static_cast<long long>(n_rows) * ((vocab + per - 1) / per) < 4LL * num_sms)) per /= 2;
    const int splits = (vocab + per - 1) / per;
    return splits < 1 ? 1 : splits > 32 ? 32 : splits;
}

size_t draft_workspace(int n_rows) { return sizeof(float4) * 2 * 32 * static_cast<size_t>(n_rows); }

cudaError_t launch_verify_drafts(DraftParams p, int num_sms, cudaStream_t stream) {
    p.splits = draft_splits(p.n_rows, p.vocab, num_sms);
    const dim3 grid(p.n_rows, p.splits, p.draft ? 2 : 1);
    if (p.n_rows > 0) {
        if (p.bf16_logits) draft_rows_kernel<bf16><<<grid, DR_THREADS, 0, stream>>>(p);
        else draft_rows_kernel<float><<<grid, DR_THREADS, 0, stream>>>(p);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    // a CTA takes 8 entries per thread at least
    p.ranks = 1;
    while (p.ranks < 8 && p.vocab > DV_THREADS * 8 * p.ranks) p.ranks *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.batch) * p.ranks);
    cfg.blockDim = dim3(DV_THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // its start under the first kernel's end
    at[0].val.programmaticStreamSerializationAllowed = 1;
    int n = 1;
    if (p.ranks > 1) {
        at[n].id = cudaLaunchAttributeClusterDimension;
        at[n].val.clusterDim.x = p.ranks;
        at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = at;
    cfg.numAttrs = n;
    return p.bf16_logits ? cudaLaunchKernelEx(&cfg, draft_verify_kernel<bf16>, p) : cudaLaunchKernelEx(&cfg, draft_verify_kernel<float>, p);
}

}  // namespace vl
