// Checking drafted tokens against the target's distribution with given random numbers.
//
// Row i of a sequence holds the logits of what follows its input token i; p = softmax(l / T), q the draft's distribution of the same row (or
// one at the drafted token).  The token x of row i + 1 is accepted iff u q(x) < p(x).  The first that is not is replaced by a draw from
// max(0, p - q), after the last one a token is drawn from p, both as the first v whose running sum exceeds s times the total.
//
// What comes out are whole numbers, so the arithmetic has to be good to the border: a draw among 10^5 tokens lies within 10^-6 of one
// often enough.  Two kernels:
//
// draft_rows_kernel, bound by HBM and by the instructions per entry: maximum and sum of exp2 in fp32 of every row that counts, divided over the vocabulary, one
// pass (64 sequences of up to 6 rows x 128256 bf16 entries, target and draft: 37 us for 146 MB, 61 % of the copy rate).
// draft_verify_kernel, a cluster per sequence, bound by issue and the fp64 pipe where it draws (the same call: 34 us, fp64 pipe 40 % busy, 2.1 of 4
// instructions a clock), by a chain of reads and barriers for small calls (9 us): joins these, accepts what is clear at fp32's error, decides the rows next to the border from
// sums in 64 bits, and draws by sums in 64 bits: over CTAs, warps, parts of a warp's share, steps, lanes and entries, at each level the last part that begins at or before
// the drawn point and is not empty.  max(0, p - q) needs both rows' totals, which the pass over them yields only at its end: it adds up p and q over the entries
// with p > q as fp32 sees it, and beside them a bound of what the entries near p = q may be worth.  Where the drawn point is not farther than that from the
// borders of its token, a second pass adds up max(0, p - q) itself (logits of 128256 entries, the draft's 0.6 away: no draw of 2560, 0.1 away: 6 in fp32, 0.01
// away: 300, within 0.001: all; 64 of them, one row each, 60 us without it, 91 - 96 with it).
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
    // Entries [j0, j0 + E) as they lie in memory, -inf outside the row.
    __device__ __forceinline__ uint4 load(int j0) const {
        if (j0 >= 0 && j0 + E <= vocab && (reinterpret_cast<uintptr_t>(base + j0) & 15u) == 0) return __ldg(reinterpret_cast<const uint4*>(base + j0));
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (sizeof(T) == 4) w[i] = __float_as_uint(in(j0 + i) ? entry(j0 + i) : -INFINITY);
            else w[i] = (__float_as_uint(in(j0 + 2 * i) ? entry(j0 + 2 * i) : -INFINITY) >> 16) | __float_as_uint(in(j0 + 2 * i + 1) ? entry(j0 + 2 * i + 1) : -INFINITY);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ bool in(int j) const { return j >= 0 && j < vocab; }
    // Entry i of what load gave
    __device__ static __forceinline__ float get(const uint4& v, int i) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        return sizeof(T) == 4 ? __uint_as_float(w[i % 4]) : i & 1 ? bf16_hi(w[i / 2 % 4]) : bf16_lo(w[i / 2 % 4]);
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

// Pairs of fp32 operations
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
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

    // the target's first blocks are on their way while the row's sequence is looked up; a draft row that nothing follows need not be there to be read
    uint4 raw[DR_UNROLL];
    constexpr uint32_t kNothing = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;  // -inf
    auto fetch = [&](int b) {
#pragma unroll
        for (int u = 0; u < DR_UNROLL; ++u) {
            raw[u] = b + u * DR_THREADS < b1 ? r.load((b + u * DR_THREADS) * E - r.off) : make_uint4(kNothing, kNothing, kNothing, kNothing);
        }
    };
    if (!draft) fetch(b0 + tid);
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
    if (draft) fetch(b0 + tid);
    const float c = greedy ? 0.f : static_cast<float>(kLog2e / static_cast<double>(temp));

    float m = -INFINITY, s = 0.f;
    int at = 0x7FFFFFFF;
    for (int b = b0 + tid; b < b1; b += DR_THREADS * DR_UNROLL) {
        uint4 now[DR_UNROLL];
#pragma unroll
        for (int u = 0; u < DR_UNROLL; ++u) now[u] = raw[u];
        fetch(b + DR_THREADS * DR_UNROLL);  // the next blocks are on their way under these
        if (greedy) {
#pragma unroll
            for (int u = 0; u < DR_UNROLL; ++u)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float v = r.get(now[u], i);
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
            for (int i = 0; i < E; ++i) top = fmaxf(top, r.get(now[u], i));
        // an entry of -inf with nothing finite before it: any finite reference does
        const float ref = top == -INFINITY ? 0.f : top;
        const uint64_t less = pack2(-ref, -ref), c2 = pack2(c, c);
        uint64_t add[2] = {0, 0};
#pragma unroll
        for (int u = 0; u < DR_UNROLL; ++u)
#pragma unroll
            for (int i = 0; i < E; i += 2) {
                float x, y;
                unpack2(mul2(add2(pack2(r.get(now[u], i), r.get(now[u], i + 1)), less), c2), x, y);
                add[i / 2 & 1] = add2(add[i / 2 & 1], pack2(exp2_approx(x), exp2_approx(y)));
            }
        float s0, s1;
        unpack2(add2(add[0], add[1]), s0, s1);
        s = (m == -INFINITY ? s : s * exp2_approx((m - ref) * c)) + (s0 + s1);
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

// exp((l - top) / T) for l <= top in 64 bits: 2^n times a polynomial for the rest, |r| <= 1/2, degree 8 through the nine Chebyshev points, relative error
// below 2e-12.  No table: reads of one in shared memory conflict (a draw of 64 sequences: 134 us with one of 256 entries).
struct Exp64 {
    double scale;  // log2 e / T
    float floor;   // differences of logits below this: 0
    // less: -top
    __device__ __forceinline__ double operator()(float l, float top, double less) const {
        // the float as a double by its bits: a conversion instruction costs as much as four additions (subnormals become
        // 2^-127 or so, infinities and NaN do not matter here)
        const int bits = __float_as_int(l);
        const double d = __hiloint2double(((bits >> 3) & 0x8FFFFFFF) + 0x38000000, bits << 29);
        // the difference first: both may be far larger than it, and scale is as large as 2^100
        const double x = d + less, big = fma(x, scale, 6755399441055744.0);  // 1.5 2^52: the nearest integer in the low bits
        const double r = fma(x, scale, -(big - 6755399441055744.0));
        double e = fma(r, 1.3255224878668817e-06, 1.5310079402249296e-05);
        e = fma(r, e, 0.00015403455852453838);
        e = fma(r, e, 0.0013333450568000645);
        e = fma(r, e, 0.009618129159402558);
        e = fma(r, e, 0.05550410941205933);
        e = fma(r, e, 0.2402265069581299);
        e = fma(r, e, 0.6931471805459335);
        e = fma(r, e, 1.0);
        e = __hiloint2double(__double2hiint(e) + (__double2loint(big) << 20), __double2loint(e));
        return l - top > floor ? e : 0.0;
    }
};

// What is drawn from: weights of a row's entries.
struct Weights {
    int kind;       // 0: p; 1: p without token x; 2: max(0, p - q); 3: the same, from the totals of a pass of kind 2
    int x;
    float pm, qm;   // the rows' maxima
    double ps, qs;  // and -1 times these
    double a, b;    // kinds 2 and 3: a e_p - b e_q, a = sum e_q, b = sum e_p
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

__device__ __forceinline__ float load_cluster32(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// The weights of block f of a row that begins at entry j0, g: the draft's (kinds 2 and 3).
template <typename T>
__device__ __forceinline__ void weights_of(const uint4& f, const uint4& g, const Exp64& ex, const Weights& w, int j0, double (&v)[Row<T>::E]) {
    constexpr int E = Row<T>::E;
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = ex(Row<T>::get(f, i), w.pm, w.ps);
    if (w.kind == 1) {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (j0 + i == w.x) v[i] = 0.0;
    } else if (w.kind >= 2) {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = fmax(0.0, __dsub_rn(__dmul_rn(w.a, v[i]), __dmul_rn(w.b, ex(Row<T>::get(g, i), w.qm, w.qs))));  // (no fma: 0 where p = q)
    }
}

template <typename T>
__global__ void __launch_bounds__(DV_THREADS) draft_verify_kernel(const DraftParams p) {
    constexpr int E = Row<T>::E;
    __shared__ double warp_tot[4][DV_WARPS];
    __shared__ double cta_tot[2][4];  // used in turn
    __shared__ float warp_near[DV_WARPS], cta_near[2];
    __shared__ float sm_sure;  // not 0: the token drawn is the right one
    __shared__ double part_tot[DV_WARPS];
    __shared__ float sm_pm[kDraftMaxRows], sm_ps[kDraftMaxRows], sm_qm[kDraftMaxRows], sm_qs[kDraftMaxRows];
    __shared__ int sm_code[kDraftMaxRows], sm_arg[kDraftMaxRows];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ranks = p.ranks, rank = ranks > 1 ? static_cast<int>(cluster_ctarank()) : 0, b = blockIdx.x / ranks;
    const SeqRows s = seq_rows(p, b);
    const float temp = temp_of(p, b);
    const bool greedy = temp == 0.f;
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
    Exp64 ex;
    ex.scale = greedy ? 1.0 : kLog2e / static_cast<double>(temp);
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
            sm_qs[i] = qs;
        }
    }
    __syncthreads();

    int stop = 0;  // row that is drawn from, once it is known

    // ---- sums in 64 bits over the cluster
    const int blocks = (p.vocab + E - 1) / E + 1;  // of any row, whatever its alignment
    const int per_cta = (blocks + ranks - 1) / ranks, per_warp = (per_cta + DV_WARPS - 1) / DV_WARPS;
    const int wb0 = rank * per_cta + warp * per_warp;
    const int wb1 = min(min(wb0 + per_warp, (rank + 1) * per_cta), blocks);
    int turn = 0;
    // One pass over a row in 64 bits.  Per warp, per CTA and over the cluster: 0 = sum of e_p (without token x for kind 1); for kind 2 that and 1 = sum of e_q
    // over the entries with p <= q, 2 and 3 the same over those with p > q, as fp32 sees it (from differences to the largest logits); for kind 3 the sum of max(0, p - q).
    //
    // `err` bounds what that may be wrong by, of all parts together.  log2 p = (l - max) c - log2(sum): the difference, the product and the logarithm
    // are each rounded by at most 2^-23 of log2 p (c's own error is common to p and q), those of p and q together by less than 6e-7 |log2 p|; with both sums right
    // to 2.5e-6 of their ratio, which the pass itself shows, an entry is on the wrong side only where fp32 sees p and q within 4e-6 + 6e-7 |log2 p| of one another, and |p - q| is
    // at most that times p.
    Weights w;
    double total[4];  // of the row: 0 sum of e_p, 1 of e_q, 2 and 3 over p > q
    double cta_part = 0.0;  // lane 4 r + i: sum i of CTA r
    double err = 0.0;
    // joins the threads' sums v; bounded: and near, the sum of p times its distance from q, into err
    auto join = [&](const double (&v)[4], bool bounded, float near) {
        __syncthreads();  // the sums of an earlier pass have been read
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const double sum = warp_sum64(v[q]);
            if (lane == 0) warp_tot[q][warp] = sum;
        }
        if (bounded) {
            near = warp_sum(near);
            if (lane == 0) warp_near[warp] = near;
        }
        __syncthreads();
        turn ^= 1;
        if (warp < 4) {  // one sum each; the order is the same everywhere
            double sum = lane < DV_WARPS ? warp_tot[warp][lane] : 0.0;
            sum = warp_sum64(sum);
            if (lane == 0) cta_tot[turn][warp] = sum;
        } else if (warp == 4 && bounded) {
            const float sum = warp_sum(lane < DV_WARPS ? warp_near[lane] : 0.f);
            if (lane == 0) cta_near[turn] = sum;
        }
        if (ranks > 1) {
            __syncwarp();
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
        cta_part = 0.0;
        if (lane < 4 * ranks) cta_part = ranks > 1 ? load_cluster64(map_to_cta(smem_u32(&cta_tot[turn][lane & 3]), lane >> 2)) : cta_tot[turn][lane];
        float of_cta = 0.f;
        if (bounded && lane < ranks) of_cta = ranks > 1 ? load_cluster32(map_to_cta(smem_u32(&cta_near[turn]), lane)) : cta_near[turn];
        err = bounded ? warp_sum(of_cta) : 0.f;
        double sum = cta_part;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
#pragma unroll
        for (int q = 0; q < 4; ++q) total[q] = __shfl_sync(0xFFFFFFFFu, sum, q);
        total[0] += total[2];
        total[1] += total[3];
    };
    // A pass over row `stop`; one of kind 3 follows one of kind 2 over the same row.
    auto pass = [&](int kind, int x) {
        const Row<T> rp(p.target, p.target_stride, s.row0 + stop, p.vocab), rq(p.draft ? p.draft : p.target, p.draft ? p.draft_stride : p.target_stride, s.row0 + stop, p.vocab);
        w.kind = kind;
        w.x = x;
        w.pm = sm_pm[stop];
        w.qm = sm_qm[stop];
        w.ps = -static_cast<double>(w.pm);
        w.qs = -static_cast<double>(w.qm);
        double v[4] = {0.0, 0.0, 0.0, 0.0}, near = 0.0;
        // blocks are fetched two steps ahead
        auto fetch = [&](int k, uint4& f, uint4& g) {
            const int j0 = k < wb1 ? k * E - rp.off : p.vocab;
            f = rp.load(j0);
            if (kind >= 2) g = rq.load(j0);
        };
        uint4 f0, f1, g0 = make_uint4(0u, 0u, 0u, 0u), g1 = g0;
        fetch(wb0 + lane, f0, g0);
        fetch(wb0 + lane + 32, f1, g1);
        // (a loop for kind 2 alone: 64 sequences over 128256 entries took 83 us with one for all kinds, 74 then)
        if (kind == 2) {
            const float kp = -log2f(sm_ps[stop]), kq = -log2f(sm_qs[stop]);
            for (int k = wb0 + lane; k - lane < wb1; k += 32) {
                const uint4 f = f0, g = g0;
                f0 = f1;
                g0 = g1;
                fetch(k + 64, f1, g1);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float lp = rp.get(f, e), lq = rq.get(g, e);
                    const double ep = ex(lp, w.pm, w.ps), eq = ex(lq, w.qm, w.qs);
                    const float log_p = fmaf(lp - w.pm, c, kp), diff = log_p - fmaf(lq - w.qm, c, kq), eps = fmaf(-6e-7f, log_p, 4e-6f);
                    if (fabsf(diff) < eps) near += ep * static_cast<double>(eps);
                    if (diff > 0.f) {
                        v[2] += ep;
                        v[3] += eq;
                    } else {
                        v[0] += ep;
                        v[1] += eq;
                    }
                }
            }
        } else {
            for (int k = wb0 + lane; k - lane < wb1; k += 32) {
                const uint4 f = f0, g = g0;
                f0 = f1;
                g0 = g1;
                fetch(k + 64, f1, g1);
                double x[E];
                weights_of<T>(f, g, ex, w, k * E - rp.off, x);
#pragma unroll
                for (int e = 0; e < E; ++e) v[0] += x[e];
            }
        }
        // (up to float, and not to 0 from above it)
        join(v, kind == 2, near > 0.0 ? fmaxf(__double2float_ru(near), 1e-37f) : 0.f);
        if (kind == 2) {
            w.a = total[1];
            w.b = total[0];
            // (a p in units of a e_p; 2^x - 1 is less than 0.75 x up to x = 0.2, and where 4e-6 + 6e-7 |log2 p| is more e_p is 0)
            const double of_p = total[1] * static_cast<double>(sm_ps[stop]), of_q = total[0] * static_cast<double>(sm_qs[stop]);
            err = fabs(of_p - of_q) <= 2.5e-6 * of_q ? 0.75 * total[1] * err : INFINITY;
        }
    };
    // the weight of a part of the row from its four sums
    auto weight = [&](double e, double pa, double qa) { return w.kind == 2 ? fmax(0.0, __dsub_rn(__dmul_rn(w.a, pa), __dmul_rn(w.b, qa))) : e; };

    // ---- how many are accepted, and the draw behind them.  There is one place for all passes, because calls find the code cold between others: one sequence
    // after 1 ms of other kernels takes 16 - 18 us, 22 - 26 with the pass compiled where it is called.
    int code, kind, drafted;
    auto walk = [&] {  // to the first row that is not clearly accepted (the last one's code is never 0), and the pass that it takes
        while (sm_code[stop] == 0) ++stop;
        code = sm_code[stop];
        drafted = code == 1 || code == 2 ? __ldg(p.tokens + s.row0 + stop + 1) : -1;
        kind = code == 4 ? 0 : p.draft ? 2 : code == 2 ? 0 : 1;
    };
    walk();
    bool written = false, made = false;  // made: there is a pass to draw from already
    const double u = fmin(fmax(static_cast<double>(__ldg(p.sample_u + b)), 0.0), 1.0);
    for (;;) {
        if (code != 2 && !written) {
            written = true;
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
                    __syncwarp();  // (whole warps arrive)
                    cluster_arrive();
                    cluster_wait();
                }
                return;
            }
        }
        if (!made) pass(kind, drafted);
        made = false;
        const Row<T> rp(p.target, p.target_stride, s.row0 + stop, p.vocab), rq(p.draft ? p.draft : p.target, p.draft ? p.draft_stride : p.target_stride, s.row0 + stop, p.vocab);
        if (code == 2) {  // decided from sums in 64 bits
            const double ep = ex(rp.entry(drafted), w.pm, w.ps), au = static_cast<double>(__ldg(p.accept_u + s.row0 + stop + 1));
            if (p.draft ? au * ex(rq.entry(drafted), w.qm, w.qs) * total[0] < ep * total[1] : au * total[0] < ep) {
                ++stop;
                walk();
            } else {
                code = 1;
                if (p.draft) made = true;
                else kind = 1;
            }
            continue;
        }
        const double all = weight(total[0], total[2], total[3]);
        if (err > 0.0 && !(all > 2.0 * p.vocab * err)) {  // as good as every point would be too near a border
            kind = 3;
            continue;
        }
        if (!(all > 0.0) && kind != 0) {  // p nowhere above q (they are the same and the number was 1): drawn from p
            kind = 0;
            continue;
        }
        const double point = u * all;
        // the last CTA that begins at or before the point and is not empty
        int owner = 0;
        double before = 0.0, base = 0.0;
        for (int r = 0; r < ranks; ++r) {
            const double v = weight(__shfl_sync(0xFFFFFFFFu, cta_part, 4 * r), __shfl_sync(0xFFFFFFFFu, cta_part, 4 * r + 2), __shfl_sync(0xFFFFFFFFu, cta_part, 4 * r + 3));
            if (v > 0.0 && before <= point) {
                owner = r;
                base = before;
            }
            before += v;
        }
        if (owner == rank) {
            int ow = 0;
            double at = base, start = base;
            const double mine = lane < DV_WARPS ? weight(warp_tot[0][lane], warp_tot[2][lane], warp_tot[3][lane]) : 0.0;
            for (int k = 0; k < DV_WARPS; ++k) {
                const double v = __shfl_sync(0xFFFFFFFFu, mine, k);
                if (v > 0.0 && at <= point) {
                    ow = k;
                    start = at;
                }
                at += v;
            }
            // that warp's blocks again, dealt over all warps in whole steps of 32, and the one with the point
            const int o0 = rank * per_cta + ow * per_warp, o1 = min(min(o0 + per_warp, (rank + 1) * per_cta), blocks);
            const int per_part = (o1 - o0 + DV_WARPS * 32 - 1) / (DV_WARPS * 32) * 32, k_first = o0 + warp * per_part, k_last = min(k_first + per_part, o1);
            double x[E], sum = 0.0;
            auto step = [&](int k) {  // x = the weights of block k
                double v = 0.0;
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = 0.0;
                const int j0 = k * E - rp.off;
                if (k < k_last) weights_of<T>(rp.load(j0), kind >= 2 ? rq.load(j0) : make_uint4(0u, 0u, 0u, 0u), ex, w, j0, x);
#pragma unroll
                for (int e = 0; e < E; ++e) v += x[e];
                return v;
            };
            for (int k0 = k_first; k0 < k_last; k0 += 32) sum += step(k0 + lane);
            const double part = warp_sum64(sum);
            if (lane == 0) part_tot[warp] = part;
            if (tid == 0) sm_sure = 0.f;
            __syncthreads();
            // (none where the warp's share came out above 0 by what fp32 mistook: then it is not sure)
            int op = -1;
            double run = start;
            at = start;
            const double parts = lane < DV_WARPS ? part_tot[lane] : 0.0;
            for (int k = 0; k < DV_WARPS; ++k) {
                const double v = __shfl_sync(0xFFFFFFFFu, parts, k);
                if (v > 0.0 && at <= point) {
                    op = k;
                    run = at;
                }
                at += v;
            }
            if (warp == op) {
                int token = -1;
                double begin_of = 0.0, size_of = 0.0;
                for (int k0 = k_first; k0 < k_last; k0 += 32) {
                    const int k = k0 + lane;
                    if (per_part > 32) sum = step(k);  // (else it is still there)
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
                        double r = begin, at_tok = 0.0, of_tok = 0.0;
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            if (x[e] > 0.0 && r <= point) {
                                tok = k * E - rp.off + e;
                                at_tok = r;
                                of_tok = x[e];
                            }
                            r += x[e];
                        }
                        const int from = 31 - __clz(who);
                        token = __shfl_sync(0xFFFFFFFFu, tok, from);
                        begin_of = __shfl_sync(0xFFFFFFFFu, at_tok, from);
                        size_of = __shfl_sync(0xFFFFFFFFu, of_tok, from);
                    }
                    run += __shfl_sync(0xFFFFFFFFu, incl, 31);
                }
                // the point and where the token begins are off by at most err each
                const bool sure = err == 0.0 || (begin_of + 2.0 * err <= point && point + 2.0 * err < begin_of + size_of);
                if (lane == 0 && sure) {
                    sm_sure = 1.f;
                    p.out_tokens[s.row0 + stop] = token;
                    if (p.logp) p.logp[s.row0 + stop] = token < 0 ? 0.f : static_cast<float>(kLn2) * ((rp.entry(token) - w.pm) * c - log2f(sm_ps[stop]));
                }
            }
        }
        if (err == 0.0) break;
        __syncwarp();
        bool sure;
        if (ranks > 1) {
            cluster_arrive();
            cluster_wait();
            sure = load_cluster32(map_to_cta(smem_u32(&sm_sure), owner)) != 0.f;
        } else {
            __syncthreads();
            sure = sm_sure != 0.f;
        }
        if (sure) break;
        kind = 3;
    }
    if (ranks > 1) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
}

}  // namespace

// Parts that a row is divided into: 65536 entries each where that gives every SM four, down to 1024 where it does not; a lane joins each.
static int draft_splits(int n_rows, int vocab, int num_sms) {
    int per = 65536;
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
    // a CTA takes 4096 entries of a row at least; larger clusters as long as all CTAs run at once, one per SM
    // (64 sequences over 128256 entries: two waves of clusters of four take 10 us longer than clusters of two)
    p.ranks = 1;
    while (p.ranks < 8 && p.vocab > 4096 * p.ranks && static_cast<long long>(p.batch) * p.ranks * 2 <= num_sms) p.ranks *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.batch) * p.ranks);
    cfg.blockDim = dim3(DV_THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    int n = 0;
    if (p.n_rows > 0) {  // its start under the first kernel's end
        at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
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
