// The pages of a paged cache: freeing, handing out, forking, compacting -- sm_100a device code.
//
// State: refs[p] = table entries that name page p (0: free), and the block tables themselves, -1 where a
// sequence has no page.  Pages are handed out lowest first, in the order of the requests, found by a scan
// of refs: the result depends on the state alone, never on the order in which CTAs run.  The metadata is a
// few hundred kilobytes at most and costs one CTA's scan; what takes time is the copying of pages, every
// byte read once and written once.
#pragma once
#include "lagkv_attend_kernels.cuh"

namespace lagkv {

constexpr int kPageThreads = 256;
constexpr int kScanThreads = 512;
constexpr int kCopyVectors = 4;                                   // 16-byte vectors per thread and step
constexpr int kCopySlice = kPageThreads * kCopyVectors;           // vectors of one CTA step

struct PageParams {
    uint8_t* K;
    uint8_t* V;
    int32_t* table;      // [B, max_blocks]
    int32_t* refs;       // [num_pages]
    int32_t* status;
    int32_t* arrived;    // CTAs that have counted (zero between calls)
    int32_t* work;       // per-sequence / per-pair numbers
    int32_t* list;       // pages found: [0, num_pages) one list, [num_pages, 2 num_pages) another
    long long num_pages;
    long long page_stride, sh, ss;  // bytes
    int B, H, max_blocks, page_shift, vpr;
    bool dense;          // a page is one run of H * page_size * vpr vectors
};

// inclusive scan over the CTA; `sums` [32] shared; returns this thread's inclusive value and the total
__device__ __forceinline__ int cta_scan(int v, int* sums, int* total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, nw = blockDim.x >> 5;
    int inc = v;
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(~0u, inc, o);
        if (lane >= o) inc += u;
    }
    __syncthreads();
    if (lane == 31) sums[w] = inc;
    __syncthreads();
    int part = lane < nw ? sums[lane] : 0;  // every warp scans the warps' sums itself
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(~0u, part, o);
        if (lane >= o) part += u;
    }
    const int all = __shfl_sync(~0u, part, 31), before = w ? __shfl_sync(~0u, part, w - 1) : 0;
    *total = all;
    return before + inc;
}

// The lowest `want` pages with refs == 0, in ascending order, into list; returns how many there are (at
// least `want` if there are that many; the scan ends once it has found them).
__device__ __forceinline__ long long find_free(const PageParams& P, long long want, int* sums) {
    constexpr int PER = 8;
    long long found = 0;
    for (long long p0 = 0; p0 < P.num_pages && found < want; p0 += (long long)blockDim.x * PER) {
        const long long mine = p0 + (long long)threadIdx.x * PER;
        unsigned bits = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (mine + i < P.num_pages && P.refs[mine + i] == 0) bits |= 1u << i;
        int total;
        const int n = __popc(bits);
        long long at = found + cta_scan(n, sums, &total) - n;
        for (; bits; bits &= bits - 1, ++at)
            if (at < want) P.list[at] = int(mine + __ffs(int(bits)) - 1);
        found += total;
    }
    return found;
}

// True in the last CTA of the grid to get here; what the others wrote before is visible to it.
__device__ __forceinline__ bool last_cta(int32_t* arrived, int* flag) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        *flag = atomicAdd(arrived, 1) == int(gridDim.x) - 1;
        if (*flag) *arrived = 0;
    }
    __syncthreads();
    const bool last = *flag != 0;
    if (last) __threadfence();
    return last;
}

// ------------------------------------------------------------------------------------ release
__global__ void __launch_bounds__(kPageThreads)
lagkv_pages_release_kernel(const PageParams P, const int32_t* __restrict__ keep_len) {
    const long long total = (long long)P.B * P.max_blocks;
    for (long long i = blockIdx.x * (long long)kPageThreads + threadIdx.x; i < total; i += (long long)gridDim.x * kPageThreads) {
        const int b = int(i / P.max_blocks), j = int(i % P.max_blocks);
        const int keep = __ldg(keep_len + b);
        if (keep < 0 || keep > ((long long)P.max_blocks << P.page_shift)) {
            if (j == 0) record_status(P.status, ST_EINVAL, b);
            continue;
        }
        const int p = P.table[i];
        if (p < 0 || ((long long)j << P.page_shift) < keep) continue;
        if (p >= P.num_pages) {
            record_status(P.status, ST_EINVAL, b);
            continue;
        }
        if (atomicSub(P.refs + p, 1) <= 0) {  // counted by nobody: put it back, keep the entry
            atomicAdd(P.refs + p, 1);
            record_status(P.status, ST_EINVAL, b);
            continue;
        }
        P.table[i] = -1;
    }
}

// ------------------------------------------------------------------------------------ reserve
// One CTA per sequence counts the pages it lacks; the last to arrive finds as many free ones and deals
// them out in the order (sequence, block).  Too few: nothing changes.  work[b] = pages lacked, then the
// offset into the list.
__global__ void __launch_bounds__(kScanThreads)
lagkv_pages_reserve_kernel(const PageParams P, const int32_t* __restrict__ want_len) {
    __shared__ int sums[32];
    __shared__ int flag;
    const int b = blockIdx.x, tid = threadIdx.x;
    {
        const int want = want_len[b];
        const long long room = (long long)P.max_blocks << P.page_shift;
        int lack = 0;
        if (want < 0 || want > room) {
            if (tid == 0) record_status(P.status, ST_EINVAL, b);
        } else {
            const int nb = (want + (1 << P.page_shift) - 1) >> P.page_shift;
            for (int j = tid; j < nb; j += kScanThreads) lack += P.table[(long long)b * P.max_blocks + j] < 0;
        }
        int total;
        cta_scan(lack, sums, &total);
        if (tid == 0) P.work[b] = total;
    }
    if (!last_cta(P.arrived, &flag)) return;
    long long need = 0;
    for (int b0 = 0; b0 < P.B; b0 += kScanThreads) {
        const int i = b0 + tid;
        const int n = i < P.B ? __ldcg(P.work + i) : 0;
        int total;
        const int inc = cta_scan(n, sums, &total);
        // -1: nothing to do for this sequence
        if (i < P.B) P.work[i] = n ? int(min(need + inc - n, 0x7fffffffll)) : -1;
        need += total;
    }
    if (need == 0) return;
    if (find_free(P, need, sums) < need) {
        if (tid == 0) record_status(P.status, ST_ECAPACITY, -1);
        return;
    }
    __syncthreads();
    const int lane = tid & 31;
    for (int i = tid >> 5; i < P.B; i += kScanThreads / 32) {
        int at = P.work[i];
        if (at < 0) continue;
        const int nb = (want_len[i] + (1 << P.page_shift) - 1) >> P.page_shift;
        int32_t* row = P.table + (long long)i * P.max_blocks;
        for (int j0 = 0; j0 < nb; j0 += 32) {
            const int j = j0 + lane;
            const bool lack = j < nb && row[j] < 0;
            const unsigned m = __ballot_sync(~0u, lack);
            if (lack) {
                const int p = P.list[at + __popc(m & ((1u << lane) - 1))];
                row[j] = p;
                P.refs[p] = 1;
            }
            at += __popc(m);
        }
    }
}

// ------------------------------------------------------------------------------------ fork
// Numbers of a pair in work: [0] copies before it (-1: refused), [1] its pages, [2] of these shared, [3]
// seq_len, [4] static_len; behind the pairs the first pair that names each sequence as its target, and
// one word for the number of copies.
constexpr int kPairWords = 5;

// One CTA per pair looks at the tables; the last to arrive numbers the copies and finds their pages.
__global__ void __launch_bounds__(kScanThreads)
lagkv_pages_fork_plan_kernel(const PageParams P, const int32_t* __restrict__ seq_len, const int32_t* __restrict__ static_len,
                             const int32_t* __restrict__ src, const int32_t* __restrict__ dst) {
    __shared__ int sums[32];
    __shared__ int flag;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int i = blockIdx.x, tid = threadIdx.x, n = gridDim.x;
    int32_t* w = P.work + (long long)i * kPairWords;
    int32_t* owner = P.work + (long long)P.B * kPairWords;
    {
        const int s = src[i], d = dst[i];
        bool bad = s < 0 || s >= P.B || d < 0 || d >= P.B;
        int len = 0, fixed = 0, used = 0, shared = 0;
        if (!bad) {
            len = seq_len[s];
            fixed = static_len[s];
            bad = len < 0 || len > ((long long)P.max_blocks << P.page_shift) || fixed < 0;
        }
        if (!bad) {
            used = (len + (1 << P.page_shift) - 1) >> P.page_shift;
            shared = min(len, fixed) >> P.page_shift;
            for (int j = tid; j < P.max_blocks; j += kScanThreads) {
                if (P.table[(long long)d * P.max_blocks + j] >= 0) bad = true;  // the target holds pages
                if (j < used) {
                    const int p = P.table[(long long)s * P.max_blocks + j];
                    if (p < 0 || p >= P.num_pages || P.refs[p] < 1) bad = true;
                }
            }
        }
        bad = __syncthreads_or(bad);
        if (tid == 0) {
            w[0] = bad ? -1 : used - shared;
            w[1] = used;
            w[2] = shared;
            w[3] = len;
            w[4] = fixed;
        }
    }
    if (!last_cta(P.arrived, &flag)) return;
    // of pairs with the same target the first counts
    for (int b = tid; b < P.B; b += kScanThreads) owner[b] = 0x7fffffff;
    __syncthreads();
    for (int k = tid; k < n; k += kScanThreads)
        if (__ldcg(P.work + (long long)k * kPairWords) >= 0) atomicMin(owner + dst[k], k);
    __syncthreads();
    long long need = 0;
    for (int k0 = 0; k0 < n; k0 += kScanThreads) {
        const int k = k0 + tid;
        int c = k < n ? __ldcg(P.work + (long long)k * kPairWords) : 0;
        const bool bad = k < n && (c < 0 || owner[dst[k]] != k);
        if (bad) {
            record_status(P.status, ST_EINVAL, k);
            c = 0;
        }
        int total;
        const int inc = cta_scan(c, sums, &total);
        if (k < n) P.work[(long long)k * kPairWords] = bad ? -1 : int(min(need + inc - c, 0x7fffffffll));
        need += total;
    }
    const bool fits = need == 0 || find_free(P, need, sums) >= need;
    if (!fits && tid == 0) record_status(P.status, ST_ECAPACITY, -1);
    __syncthreads();
    // the pages to copy, in the order of those found for them
    for (int k = tid >> 5; fits && k < n; k += kScanThreads / 32) {
        const int32_t* u = P.work + (long long)k * kPairWords;
        if (u[0] < 0) continue;
        for (int j = __ldcg(u + 2) + (tid & 31); j < __ldcg(u + 1); j += 32)
            P.list[P.num_pages + u[0] + j - __ldcg(u + 2)] = P.table[(long long)src[k] * P.max_blocks + j];
    }
    if (tid == 0) owner[P.B] = fits ? int(need) : -1;  // copies to make; -1: too few free pages, nothing changes
}

// Vector v of page p of one tensor.
__device__ __forceinline__ uint4* page_vector(const PageParams& P, uint8_t* X, int p, int v) {
    uint8_t* page = X + (long long)p * P.page_stride;
    if (P.dense) return reinterpret_cast<uint4*>(page) + v;
    const int rows = 1 << P.page_shift, r = v / P.vpr, c = v % P.vpr;
    return reinterpret_cast<uint4*>(page + (long long)(r / rows) * P.sh + (long long)(r & (rows - 1)) * P.ss) + c;
}
// One slice of one page of one tensor: item = (copy, tensor, slice).
__device__ __forceinline__ void copy_slice(const PageParams& P, int from, int to, int which, int slice, int vectors) {
    uint8_t* X = which ? P.V : P.K;
    uint4 v[kCopyVectors];
    const int v0 = slice * kCopySlice + threadIdx.x;
#pragma unroll
    for (int k = 0; k < kCopyVectors; ++k)
        if (v0 + k * kPageThreads < vectors) v[k] = __ldcs(page_vector(P, X, from, v0 + k * kPageThreads));
#pragma unroll
    for (int k = 0; k < kCopyVectors; ++k)
        if (v0 + k * kPageThreads < vectors) *page_vector(P, X, to, v0 + k * kPageThreads) = v[k];
}

__global__ void __launch_bounds__(kPageThreads)
lagkv_pages_fork_kernel(const PageParams P, int32_t* seq_len, int32_t* static_len, const int32_t* __restrict__ src,
                        const int32_t* __restrict__ dst, int n) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int copies = P.work[(long long)P.B * kPairWords + P.B];
    if (copies < 0) return;
    // tables and lengths: the first CTAs, a pair at a time
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
        const int32_t* w = P.work + (long long)i * kPairWords;
        if (w[0] < 0) continue;
        const int32_t* from = P.table + (long long)src[i] * P.max_blocks;
        int32_t* to = P.table + (long long)dst[i] * P.max_blocks;
        for (int j = threadIdx.x; j < w[1]; j += kPageThreads) {
            if (j < w[2]) {
                const int p = from[j];
                to[j] = p;
                atomicAdd(P.refs + p, 1);
            } else {
                const int p = P.list[w[0] + j - w[2]];
                to[j] = p;
                P.refs[p] = 1;
            }
        }
        if (threadIdx.x == 0) {
            seq_len[dst[i]] = w[3];
            static_len[dst[i]] = w[4];
        }
    }
    const int vectors = (P.H << P.page_shift) * P.vpr, slices = (vectors + kCopySlice - 1) / kCopySlice;
    const long long items = 2ll * copies * slices;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int slice = int(it % slices), which = int(it / slices & 1), c = int(it / slices >> 1);
        copy_slice(P, P.list[P.num_pages + c], P.list[c], which, slice, vectors);
    }
}

// ------------------------------------------------------------------------------------ compact
// One CTA: counts the live pages, then lists the free ones below that number (list) and the live ones at
// or above it (list + num_pages), both ascending, and turns work into the new names of all pages (-1: not
// live).  work[0] = pages to move, then the names.
__global__ void __launch_bounds__(kScanThreads)
lagkv_pages_compact_plan_kernel(const PageParams P, int32_t* live_out) {
    __shared__ int sums[32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int PER = 8;
    const int tid = threadIdx.x;
    long long live = 0;
    int mine = 0;
    for (long long p = tid; p < P.num_pages; p += kScanThreads) mine += P.refs[p] > 0;
    int total;
    cta_scan(mine, sums, &total);
    live = total;
    long long holes = 0, movers = 0;
    for (long long p0 = 0; p0 < P.num_pages; p0 += (long long)kScanThreads * PER) {
        const long long at = p0 + (long long)tid * PER;
        unsigned hole = 0, mover = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const long long p = at + i;
            if (p < P.num_pages) {
                const bool used = P.refs[p] > 0;
                if (p < live && !used) hole |= 1u << i;
                if (p >= live && used) mover |= 1u << i;
                P.work[1 + p] = p < live && used ? int(p) : -1;
            }
        }
        int nh, nm;
        long long h = holes + cta_scan(__popc(hole), sums, &nh) - __popc(hole);
        long long m = movers + cta_scan(__popc(mover), sums, &nm) - __popc(mover);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (hole >> i & 1) P.list[h++] = int(at + i);
            if (mover >> i & 1) P.list[P.num_pages + m++] = int(at + i);
        }
        holes += nh;
        movers += nm;
    }
    __syncthreads();
    // as many holes below `live` as live pages at or above it
    for (long long i = tid; i < movers; i += kScanThreads) P.work[1 + P.list[P.num_pages + i]] = P.list[i];
    if (tid == 0) {
        P.work[0] = int(movers);
        *live_out = int(live);
    }
}

__global__ void __launch_bounds__(kPageThreads)
lagkv_pages_compact_kernel(const PageParams P) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int moves = P.work[0];
    const long long stride = (long long)gridDim.x * kPageThreads, first = blockIdx.x * (long long)kPageThreads + threadIdx.x;
    for (long long i = first; i < (long long)P.B * P.max_blocks; i += stride) {
        const int p = P.table[i];
        if (p < 0) continue;
        const int to = p < P.num_pages ? P.work[1 + p] : -1;
        // a page that is not live: the number may be another sequence's page from now on
        if (to < 0) record_status(P.status, ST_EINVAL, int(i / P.max_blocks));
        if (to != p) P.table[i] = to;
    }
    for (long long i = first; i < moves; i += stride) {
        const int from = P.list[P.num_pages + i], to = P.list[i];
        P.refs[to] = P.refs[from];
        P.refs[from] = 0;
    }
    const int vectors = (P.H << P.page_shift) * P.vpr, slices = (vectors + kCopySlice - 1) / kCopySlice;
    const long long items = 2ll * moves * slices;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int slice = int(it % slices), which = int(it / slices & 1), c = int(it / slices >> 1);
        copy_slice(P, P.list[P.num_pages + c], P.list[c], which, slice, vectors);
    }
}

}  // namespace lagkv
