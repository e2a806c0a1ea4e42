// Keeping the accepted path of a tree of drafted tokens: its rows move down inside the cache, in place.
#pragma once
#include "lagkv_attend_kernels.cuh"

namespace lagkv {

constexpr int kCommitThreads = 512;

// One CTA per sequence.  Row j of the path comes from row accepted[j] >= j of the draft and the path
// ascends, so what a pass of rows [j0, j1) overwrites (rows below j1) no later pass reads: each pass
// loads all of its vectors, waits for the CTA, then stores.  A few rows of 256 bytes per head: bound by
// one load-store round trip, a single launch.
__global__ void __launch_bounds__(kCommitThreads)
lagkv_tree_commit_kernel(const AttendParams P, uint8_t* K, uint8_t* V, int vpr, int32_t* seq_len,
                         const int32_t* __restrict__ accepted, const int32_t* __restrict__ n_accepted) {
    __shared__ int path[64];
    const int b = blockIdx.x, tid = threadIdx.x;
    const int len = seq_len[b], n = n_accepted[b];
    const int draft = P.draft_len ? P.draft_len[b] : len == 0 ? 0 : P.T, base = len - draft;  // an empty slot of the batch is no error
    bool bad = len < 0 || len > P.S_cap || draft < 0 || draft > P.T || draft > len || n < 0 || n > draft;
    if (!bad && tid < n) {
        const int a = accepted[(long long)b * P.T + tid];
        path[tid] = a;
        if (a < 0 || a >= draft) bad = true;
        if (tid > 0 && accepted[(long long)b * P.T + tid - 1] >= a) bad = true;
        // every page the path reads or writes has to lie inside the pool
        if (!bad && P.block_table != nullptr && (attend_offset(P, b, 0, (base + a) & ~15) < 0 || attend_offset(P, b, 0, (base + tid) & ~15) < 0))
            bad = true;
    }
    if (__syncthreads_or(bad)) {
        if (tid == 0) record_status(P.status, ST_EINVAL, b);
        return;
    }
    const int per_row = 2 * P.H * vpr;            // vectors of one row over both tensors and all heads
    const long long total = (long long)n * per_row;
    constexpr int BATCH = 4;                      // vectors per thread and pass
    for (long long i0 = 0; i0 < total; i0 += BATCH * kCommitThreads) {
        uint4 v[BATCH];
        uint8_t* to[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const long long i = i0 + k * kCommitThreads + tid;
            to[k] = nullptr;
            if (i < total) {
                const int j = int(i / per_row), r = int(i % per_row);
                const int h = r / (2 * vpr), which = (r / vpr) & 1, c = r % vpr;
                const int src = base + path[j], dst = base + j;
                if (src != dst) {
                    uint8_t* x = which ? V : K;
                    v[k] = *reinterpret_cast<const uint4*>(x + attend_offset(P, b, h, src & ~15) + (src & 15) * P.ss + c * 16);
                    to[k] = x + attend_offset(P, b, h, dst & ~15) + (dst & 15) * P.ss + c * 16;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
            if (to[k] != nullptr) *reinterpret_cast<uint4*>(to[k]) = v[k];
        __syncthreads();
    }
    if (tid == 0) seq_len[b] = base + n;
}

}  // namespace lagkv
