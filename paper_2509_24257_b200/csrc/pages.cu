// Pages of a paged cache between attention calls: growing and shortening sequences, sharing pages, moving them.
//
// State, all on the device: the page table, the sequences' lengths, and for every page the number of table entries that name it (0: free).  A sequence
// of n positions holds the first ceil(n / page_size) entries of its row of the table.  Every operation gives the same result whatever the timing: free pages are taken lowest
// first, by sequences in order.
//
// Planning is one CTA's work over a few thousand integers, bound by latency (64 sequences growing and shrinking, 9000 pages: 14.2 us for both calls; 21.9 with
// counts read phase by phase and holders compared by single threads).  Copies are HBM-bound and spread over the GPU in pieces of 32 KB: the number of copies is only known
// on the device, so a fixed grid walks them (24 sequences of 6000 positions, 4 layers, some in, the rest compacted: 156 us for 896 MB with the planning, 89 % of the
// copy rate).
#include "common.cuh"
#include "kernels.h"

namespace vl {

namespace {

constexpr int PL_THREADS = 1024;   // planning kernels
constexpr int PL_WARPS = PL_THREADS / 32;
constexpr int PL_SMALL = 1024;     // sequences whose plans fit shared memory
constexpr int PL_STEPS = 16;       // loads of counts in flight per thread
constexpr int CP_THREADS = 256;
constexpr int CP_LOADS = 8;        // 16-byte loads in flight per thread (the two copies of the header's example 175 us with 2, 170 with 4, 156 with 8)
constexpr int CP_PIECE = CP_THREADS * 16 * CP_LOADS;  // bytes of a page that a CTA copies at a time
constexpr int WS_HEADER = 32;      // ints: [0] number of copies, [1] first page behind those in use

__device__ __forceinline__ void raise(int* status, int code) {
    if (status) atomicCAS(status, 0, code);
}
__device__ __forceinline__ int pages_of(int len, int shift) { return static_cast<int>((static_cast<long long>(len) + (1 << shift) - 1) >> shift); }

// A sequence's length, bounded to what its row of the table holds.
__device__ __forceinline__ int bounded_len(const PagesDev& p, int b) {
    const int len = p.kv_len[b];
    const long long cap = static_cast<long long>(p.table_width) << p.page_shift;
    if (len >= 0 && len <= cap) return len;
    raise(p.status, VERILLM_DEV_ROWS_RANGE);
    return len < 0 ? 0 : static_cast<int>(cap);
}

// Inclusive sum over the block; `total` is the block's.  Two barriers.
__device__ __forceinline__ long long block_scan(long long v, long long* sm, long long* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();
    if (lane == 31) sm[warp] = v;
    __syncthreads();
    long long all = sm[lane];  // (every warp adds up the warps' sums for itself)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xFFFFFFFFu, all, o);
        if (lane >= o) all += u;
    }
    *total = __shfl_sync(0xFFFFFFFFu, all, 31);
    const long long before = __shfl_sync(0xFFFFFFFFu, all, warp > 0 ? warp - 1 : 0);
    return v + (warp > 0 ? before : 0);
}
static_assert(PL_WARPS == 32, "a lane per warp in block_scan");

// Calls found(index among those found, page) for the pages of [first, last) whose being free equals `free`, in order, until at least `most` were
// found; returns how many.  A step looks at PL_STEPS runs of PL_THREADS pages, whose counts are read together.
struct ScanScratch {
    int count[PL_STEPS][PL_WARPS], run[PL_STEPS];
};
// early: the counts of the first step where they have been read already, or null.
__device__ __forceinline__ void read_counts(const PagesDev& p, long long base, int last, bool free, int (&refs)[PL_STEPS]) {
#pragma unroll
    for (int u = 0; u < PL_STEPS; ++u) {
        const long long page = base + u * PL_THREADS + threadIdx.x;
        refs[u] = page < last ? p.refs[page] : free ? 1 : 0;
    }
}
template <typename F>
__device__ __forceinline__ int scan_pages(const PagesDev& p, int first, int last, bool free, int most, ScanScratch& sm, const int (*early)[PL_STEPS], F found) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int count = 0;
    for (long long base = first; base < last && count < most; base += PL_STEPS * PL_THREADS) {
        int refs[PL_STEPS];
        unsigned who[PL_STEPS];
        if (early && base == first) {
#pragma unroll
            for (int u = 0; u < PL_STEPS; ++u) refs[u] = (*early)[u];
        } else {
            read_counts(p, base, last, free, refs);
        }
#pragma unroll
        for (int u = 0; u < PL_STEPS; ++u) {
            who[u] = __ballot_sync(0xFFFFFFFFu, (refs[u] <= 0) == free);
            if (lane == 0) sm.count[u][warp] = __popc(who[u]);
        }
        __syncthreads();
        if (warp < PL_STEPS) {  // one warp per run: counts to places
            const int mine = sm.count[warp][lane];
            int v = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int w = __shfl_up_sync(0xFFFFFFFFu, v, o);
                if (lane >= o) v += w;
            }
            sm.count[warp][lane] = v - mine;
            if (lane == 31) sm.run[warp] = v;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PL_STEPS; ++u) {
            if (who[u] >> lane & 1u)
                found(count + sm.count[u][warp] + __popc(who[u] & ((1u << lane) - 1u)), static_cast<int>(base + u * PL_THREADS + tid));
            count += sm.run[u];
        }
        __syncthreads();  // the scratch is written again
    }
    return count;
}

// Workspace: header, then lists of max(batch, n_pages) ints each.
struct Lists {
    int *header, *src, *dst, *list, *need, *upto;
};
__host__ __device__ __forceinline__ Lists lists_of(int* ws, int batch, int n_pages) {
    const size_t most = static_cast<size_t>(batch > n_pages ? batch : n_pages) + 3 & ~static_cast<size_t>(3);
    Lists l;
    l.header = ws;
    l.src = ws + WS_HEADER;
    l.dst = l.src + most;
    l.list = l.dst + most;
    l.need = l.list + most;
    l.upto = l.need + most;
    return l;
}

// Growing.  A sequence that grows takes the lowest free pages for its new positions, and one more for a copy of its last page if that is partly
// filled and others name it too; of the holders of one such page the last keeps it where all of them grow.  Sequences are served in order up to the
// first whose need exceeds what is left.
__global__ void __launch_bounds__(PL_THREADS) reserve_kernel(const PagesDev p, const int* __restrict__ new_len, int* ws) {
    __shared__ ScanScratch sm_scan;
    __shared__ long long sm_sum[PL_WARPS];
    __shared__ int sm_count, sm_copies;
    __shared__ int sm_lists[7][PL_SMALL];
    const Lists l = lists_of(ws, p.batch, p.n_pages);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // what a usual batch needs stays in shared memory: the phases below are a chain of reads
    const bool small = p.batch <= PL_SMALL;
    int *need_of = small ? sm_lists[0] : l.need, *upto_of = small ? sm_lists[1] : l.upto;
    int *held_seq = small ? sm_lists[2] : l.src, *held_page = small ? sm_lists[3] : l.dst, *held_copy = small ? sm_lists[4] : l.list;
    const long long cap = static_cast<long long>(p.table_width) << p.page_shift;
    int early[PL_STEPS];  // read under the first phases, written only in the last
    read_counts(p, 0, p.n_pages, true, early);
    if (tid == 0) sm_count = sm_copies = 0;
    pdl_launch_dependents();
    __syncthreads();
    // sequences that would write into a page that others hold: src = sequence, dst = that page (in any order)
    for (int b = tid; b < p.batch; b += PL_THREADS) {
        const int len = bounded_len(p, b), want = new_len[b];
        int need = -1;  // does not grow
        if (want > len) {
            if (want > cap) {
                raise(p.status, VERILLM_DEV_ROWS_RANGE);
            } else {
                const int have = pages_of(len, p.page_shift);
                need = min(pages_of(want, p.page_shift) - have, p.n_pages + 1);  // (one more than there are: never served)
                if (len & ((1 << p.page_shift) - 1)) {
                    const int page = p.page_table[static_cast<size_t>(b) * p.table_width + have - 1];
                    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.n_pages)) {
                        raise(p.status, VERILLM_DEV_PAGE_RANGE);
                        need = -1;
                    } else if (p.refs[page] > 1) {
                        const int i = atomicAdd(&sm_count, 1);
                        held_seq[i] = b;
                        held_page[i] = page;
                    }
                }
            }
        }
        need_of[b] = need;
        if (small) {
            sm_lists[5][b] = len;
            sm_lists[6][b] = want;
        }
    }
    __syncthreads();
    for (int i = warp; i < sm_count; i += PL_WARPS) {
        const int b = held_seq[i], page = held_page[i];
        int same = 0, later = 0;
        for (int j = lane; j < sm_count; j += 32)
            if (held_page[j] == page) {
                ++same;
                later |= held_seq[j] > b;
            }
        same = __reduce_add_sync(0xFFFFFFFFu, same);
        later = __reduce_or_sync(0xFFFFFFFFu, later);
        if (lane == 0) held_copy[i] = same == p.refs[page] && !later ? 0 : 1;
    }
    __syncthreads();
    for (int i = tid; i < sm_count; i += PL_THREADS)
        if (held_copy[i]) need_of[held_seq[i]] = (need_of[held_seq[i]] + 1) | 0x40000000;  // with a copy
    __syncthreads();
    long long sum = 0;
    for (int b0 = 0; b0 < p.batch; b0 += PL_THREADS) {
        const int b = b0 + tid;
        const int need = b < p.batch ? need_of[b] : -1;
        long long all;
        const long long upto = sum + block_scan(need < 0 ? 0 : need & 0x3FFFFFFF, sm_sum, &all);
        if (b < p.batch) upto_of[b] = static_cast<int>(min(upto, 0x7FFFFFFFLL));
        sum += all;
    }
    const int total = static_cast<int>(min(sum, 0x7FFFFFFFLL));
    __syncthreads();  // the lists are written again
    int* list = small && total <= PL_SMALL ? sm_lists[4] : l.list;  // the free pages that are taken
    const int found = total == 0 ? 0 : scan_pages(p, 0, p.n_pages, true, total, sm_scan, &early, [&](int k, int page) {
        if (k < total) list[k] = page;
    });
    __syncthreads();
    for (int b = warp; b < p.batch; b += PL_WARPS) {
        const int code = need_of[b];
        if (code < 0) continue;
        const int need = code & 0x3FFFFFFF, upto = upto_of[b], copy = code >> 30 & 1;
        if (upto > found) {
            if (lane == 0) raise(p.status, VERILLM_DEV_NO_PAGES);
            continue;
        }
        const int len = small ? sm_lists[5][b] : max(p.kv_len[b], 0), want = small ? sm_lists[6][b] : new_len[b];  // (a length that was bounded does not grow)
        int* row = p.page_table + static_cast<size_t>(b) * p.table_width;
        const int at = pages_of(len, p.page_shift) - copy;
        if (copy && lane == 0) {
            const int old = row[at], i = atomicAdd(&sm_copies, 1);
            l.src[i] = old;
            l.dst[i] = list[upto - need];
            atomicSub(p.refs + old, 1);
        }
        __syncwarp();
        for (int k = lane; k < need; k += 32) {
            const int page = list[upto - need + k];
            row[at + k] = page;
            p.refs[page] = 1;
        }
        __syncwarp();
        if (lane == 0) p.kv_len[b] = want;
    }
    __syncthreads();
    if (tid == 0) l.header[0] = sm_copies;
}

// Shortening: the pages behind the new end are named once less.
__global__ void __launch_bounds__(128) free_kernel(const PagesDev p, const int* __restrict__ new_len) {
    const int b = blockIdx.x;
    const int len = bounded_len(p, b), want = new_len[b];
    __syncthreads();  // all have read the length
    if (want < 0) {
        if (threadIdx.x == 0) raise(p.status, VERILLM_DEV_ROWS_RANGE);
        return;
    }
    if (want >= len) return;
    const int have = pages_of(len, p.page_shift);
    for (int j = pages_of(want, p.page_shift) + threadIdx.x; j < have; j += 128) {
        const int page = p.page_table[static_cast<size_t>(b) * p.table_width + j];
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.n_pages)) raise(p.status, VERILLM_DEV_PAGE_RANGE);
        else atomicSub(p.refs + page, 1);
    }
    if (threadIdx.x == 0) p.kv_len[b] = want;
}

// Sharing: sequence dst[i], empty, gets src[i]'s entries.  snap[i]: its length, -1 where the pair is refused; lengths are set by a second kernel,
// when all pairs have been judged by what was there before.
__global__ void __launch_bounds__(128) fork_kernel(const PagesDev p, const int* __restrict__ src, const int* __restrict__ dst, int* snap) {
    __shared__ int sm_bad;
    const int i = blockIdx.x, tid = threadIdx.x;
    const int s = src[i], d = dst[i];
    if (tid == 0) sm_bad = 0;
    pdl_launch_dependents();
    __syncthreads();
    bool bad = s < 0 || s >= p.batch || d < 0 || d >= p.batch;
    if (!bad) bad = p.kv_len[d] != 0;
    for (int j = tid; j < i; j += 128) bad = bad || dst[j] == d;  // the first of them is taken
    if (bad) sm_bad = 1;
    __syncthreads();
    if (sm_bad) {
        if (tid == 0) {
            raise(p.status, VERILLM_DEV_ROWS_RANGE);
            snap[i] = -1;
        }
        return;
    }
    const int len = bounded_len(p, s), have = pages_of(len, p.page_shift);
    const int* from = p.page_table + static_cast<size_t>(s) * p.table_width;
    int* to = p.page_table + static_cast<size_t>(d) * p.table_width;
    for (int j = tid; j < have; j += 128) {
        const int page = from[j];
        to[j] = page;
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.n_pages)) raise(p.status, VERILLM_DEV_PAGE_RANGE);
        else atomicAdd(p.refs + page, 1);
    }
    if (tid == 0) snap[i] = len;
}
__global__ void __launch_bounds__(256) fork_len_kernel(const PagesDev p, const int* __restrict__ dst, const int* snap, int n) {
    pdl_wait();
    for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256)
        if (snap[i] >= 0) p.kv_len[dst[i]] = snap[i];
}

// Compacting: U pages in use; those numbered U and above go to the free ones below, lowest to lowest.  list[page] = its new number.
__global__ void __launch_bounds__(PL_THREADS) compact_kernel(const PagesDev p, int* n_used, int* ws) {
    __shared__ ScanScratch sm_scan;
    const Lists l = lists_of(ws, p.batch, p.n_pages);
    const int used = scan_pages(p, 0, p.n_pages, false, 0x7FFFFFFF, sm_scan, nullptr, [](int, int) {});
    const int holes = scan_pages(p, 0, used, true, 0x7FFFFFFF, sm_scan, nullptr, [&](int k, int page) { l.dst[k] = page; });
    __syncthreads();
    if (holes > 0) {
        scan_pages(p, used, p.n_pages, false, 0x7FFFFFFF, sm_scan, nullptr, [&](int k, int page) { l.src[k] = page; });
        __syncthreads();
        for (int i = threadIdx.x; i < holes; i += PL_THREADS) {
            const int s = l.src[i], d = l.dst[i];
            l.list[s] = d;
            p.refs[d] = p.refs[s];
            p.refs[s] = 0;
        }
    }
    if (threadIdx.x == 0) {
        l.header[0] = holes;
        l.header[1] = used;
        *n_used = used;
    }
}

struct CopyJob {
    const int *src, *dst, *count;  // count: number of pairs, on the device, or null
    int n;                         // number of pairs, with `count` what the lists hold at most
    int src_n_pages, dst_n_pages;
    int n_layers, page_bytes, scale_bytes;
    int* status;
    // compacting: rewrite the table's entries from `first` on
    int *page_table, *kv_len;
    const int *rename, *first;
    int batch, table_width, page_shift;
};

// Pieces are counted by (pair, layer, piece of a page), the last running fastest; a CTA takes every gridDim.x-th, by additions with carries: a division of
// 64-bit numbers in every thread costs more than the copy.  Where a piece lies is looked up while the one before it is on its way.
__device__ __forceinline__ void copy_pages(const CopyJob& job, const PoolSet& from, const PoolSet& to) {
    const int n = job.count ? min(__ldcg(job.count), job.n) : job.n;
    const unsigned page_pieces = (job.page_bytes + CP_PIECE - 1) / CP_PIECE, scale_pieces = (job.scale_bytes + CP_PIECE - 1) / CP_PIECE;
    const unsigned pieces = 2 * (page_pieces + scale_pieces), layers = job.n_layers;
    const unsigned step_piece = gridDim.x % pieces, step_layer = gridDim.x / pieces % layers, step_pair = gridDim.x / pieces / layers;
    unsigned piece = blockIdx.x % pieces, layer = blockIdx.x / pieces % layers;
    long long pair = blockIdx.x / pieces / layers;

    struct Place {
        const char* x;
        char* y;
        int bytes;  // 0: nothing to copy
    };
    auto place = [&] {
        Place at = {nullptr, nullptr, 0};
        if (pair >= n) return at;
        const int s = __ldcg(job.src + pair), d = __ldcg(job.dst + pair);
        if (s == -1 || d == -1) return at;
        if (static_cast<unsigned>(s) >= static_cast<unsigned>(job.src_n_pages) || static_cast<unsigned>(d) >= static_cast<unsigned>(job.dst_n_pages)) {
            if (threadIdx.x == 0) raise(job.status, VERILLM_DEV_PAGE_RANGE);
            return at;
        }
        unsigned k = piece;
        const bool value = k >= page_pieces + scale_pieces;
        if (value) k -= page_pieces + scale_pieces;
        const bool scale = k >= page_pieces;
        if (scale) k -= page_pieces;
        const char* a = scale ? (value ? from.v_scale[layer] : from.k_scale[layer]) : (value ? from.v[layer] : from.k[layer]);
        char* b = scale ? (value ? to.v_scale[layer] : to.k_scale[layer]) : (value ? to.v[layer] : to.k[layer]);
        const int bytes = scale ? job.scale_bytes : job.page_bytes, begin = static_cast<int>(k) * CP_PIECE;
        at.x = a + static_cast<size_t>(s) * bytes + begin;
        at.y = b + static_cast<size_t>(d) * bytes + begin;
        at.bytes = min(CP_PIECE, bytes - begin);
        return at;
    };
    const int o = threadIdx.x * 16;
    Place next = place();
    while (pair < n) {
        const Place at = next;
        uint4 v[CP_LOADS];
#pragma unroll
        for (int i = 0; i < CP_LOADS; ++i)
            if (o + i * CP_THREADS * 16 < at.bytes) v[i] = *reinterpret_cast<const uint4*>(at.x + o + i * CP_THREADS * 16);
        piece += step_piece;
        unsigned carry = piece >= pieces ? 1 : 0;
        if (carry) piece -= pieces;
        layer += step_layer + carry;
        carry = layer >= layers ? 1 : 0;
        if (carry) layer -= layers;
        pair += step_pair + carry;
        next = place();
#pragma unroll
        for (int i = 0; i < CP_LOADS; ++i)
            if (o + i * CP_THREADS * 16 < at.bytes) *reinterpret_cast<uint4*>(at.y + o + i * CP_THREADS * 16) = v[i];
    }
}

// Copies within one set of pools (sources and destinations are different pages), after renaming the table's entries if asked to.
__global__ void __launch_bounds__(CP_THREADS) move_pages_kernel(const CopyJob job, const PoolSet pools) {
    pdl_wait();
    if (job.rename) {
        const int first = __ldcg(job.first);
        for (int b = blockIdx.x; b < job.batch; b += gridDim.x) {
            const long long cap = static_cast<long long>(job.table_width) << job.page_shift;
            const int len = static_cast<int>(min(static_cast<long long>(max(job.kv_len[b], 0)), cap));
            int* row = job.page_table + static_cast<size_t>(b) * job.table_width;
            for (int j = threadIdx.x; j < pages_of(len, job.page_shift); j += CP_THREADS) {
                const int page = row[j];
                if (static_cast<unsigned>(page) >= static_cast<unsigned>(job.dst_n_pages)) raise(job.status, VERILLM_DEV_PAGE_RANGE);
                else if (page >= first) row[j] = __ldcg(job.rename + page);
            }
        }
    }
    copy_pages(job, pools, pools);
}
__global__ void __launch_bounds__(CP_THREADS) copy_pages_kernel(const CopyJob job, const PoolSet from, const PoolSet to) { copy_pages(job, from, to); }

CopyJob job_of(const PagesDev& p) {
    CopyJob j = {};
    j.src_n_pages = j.dst_n_pages = p.n_pages;
    j.n_layers = p.n_layers;
    j.page_bytes = p.page_bytes;
    j.scale_bytes = p.scale_bytes;
    j.status = p.status;
    return j;
}
unsigned copy_grid(const CopyJob& j, long long most, int num_sms) {
    const long long units = most * j.n_layers * 2 * ((j.page_bytes + CP_PIECE - 1) / CP_PIECE + (j.scale_bytes + CP_PIECE - 1) / CP_PIECE);
    return static_cast<unsigned>(units < 1 ? 1 : units < 16LL * num_sms ? units : 16LL * num_sms);
}
// `kernel` after the one before it in the stream, its start under that one's end.
template <typename... A>
cudaError_t launch_after(void (*kernel)(A...), unsigned grid, unsigned block, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.stream = stream;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

size_t pages_workspace(int batch, int n_pages) {
    const size_t most = (static_cast<size_t>(batch > n_pages ? batch : n_pages) + 3) & ~static_cast<size_t>(3);
    return sizeof(int) * (WS_HEADER + 5 * most);
}

cudaError_t launch_kv_reserve(const PagesDev& p, const PoolSet& pools, const int* new_len, int* ws, int num_sms, cudaStream_t stream) {
    reserve_kernel<<<1, PL_THREADS, 0, stream>>>(p, new_len, ws);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const Lists l = lists_of(ws, p.batch, p.n_pages);
    CopyJob j = job_of(p);
    j.src = l.src;
    j.dst = l.dst;
    j.count = l.header;
    j.n = p.batch;  // (a copy per sequence at most)
    return launch_after(move_pages_kernel, copy_grid(j, j.n, num_sms), CP_THREADS, stream, j, pools);
}

cudaError_t launch_kv_free(const PagesDev& p, const int* new_len, cudaStream_t stream) {
    free_kernel<<<p.batch, 128, 0, stream>>>(p, new_len);
    return cudaGetLastError();
}

cudaError_t launch_kv_fork(const PagesDev& p, const int* src, const int* dst, int n, int* ws, cudaStream_t stream) {
    const Lists l = lists_of(ws, p.batch, p.n_pages);
    fork_kernel<<<n, 128, 0, stream>>>(p, src, dst, l.list);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_after(fork_len_kernel, static_cast<unsigned>((n + 255) / 256), 256u, stream, p, dst, static_cast<const int*>(l.list), n);
}

cudaError_t launch_kv_compact(const PagesDev& p, const PoolSet& pools, int* n_used, int* ws, int num_sms, cudaStream_t stream) {
    compact_kernel<<<1, PL_THREADS, 0, stream>>>(p, n_used, ws);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const Lists l = lists_of(ws, p.batch, p.n_pages);
    CopyJob j = job_of(p);
    j.src = l.src;
    j.dst = l.dst;
    j.count = l.header;
    j.n = p.n_pages;
    j.first = l.header + 1;
    j.rename = l.list;
    j.page_table = p.page_table;
    j.kv_len = p.kv_len;
    j.batch = p.batch;
    j.table_width = p.table_width;
    j.page_shift = p.page_shift;
    return launch_after(move_pages_kernel, copy_grid(j, j.n, num_sms), CP_THREADS, stream, j, pools);
}

cudaError_t launch_kv_copy(const PagesDev& to, const PoolSet& dst_pools, const PoolSet& src_pools, int src_n_pages, const int* src, const int* dst, int n,
                           int num_sms, cudaStream_t stream) {
    CopyJob j = job_of(to);
    j.src_n_pages = src_n_pages;
    j.src = src;
    j.dst = dst;
    j.n = n;
    copy_pages_kernel<<<copy_grid(j, n, num_sms), CP_THREADS, 0, stream>>>(j, src_pools, dst_pools);
    return cudaGetLastError();
}

}  // namespace vl
