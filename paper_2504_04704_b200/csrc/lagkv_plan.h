// What the host translation units of the C ABI share: the plan, the device guard, and the checks that
// turn a caller's strides or page layout into strides in 16-bit units.
#pragma once
#include "lagkv.h"

#include <atomic>
#include <cstring>
#include <cuda_runtime.h>
#include <mutex>

// bytes per cache element of a storage format (enum lagkv_dtype)
inline int elem_bytes(int dtype) { return dtype == LAGKV_DTYPE_FP8_E4M3 ? 1 : 2; }
inline size_t row_bytes(const lagkv_config& c) { return size_t(c.D) * elem_bytes(c.dtype); }

struct Shape {
    int kidx;         // index into kKernels
    int stages;       // ring depth per streaming warp
    int ctas_per_sm;  // grid sizing for prefill
    size_t smem;      // dynamic shared memory
};

struct lagkv_plan_s {
    lagkv_config cfg;
    int k;
    int sm_count;
    int max_smem_optin;
    Shape pre;        // kernel used by lagkv_compress_prefill
    Shape pair;       // pair kernel, preferred for short partitions with enough of them (kidx < 0: none)
    bool tuned;       // lagkv_plan_tune() fixed the prefill kernel: no switching by size
    Shape app;        // uniform kernel of lagkv_compress_append (any number of partitions per call)
    Shape app_pair;   // one-partition appends: a cluster of two CTAs per unit (kidx < 0: none)
    int app_pair_res_tiles;  // tiles of the window a CTA keeps in shared memory
    int app_pair_splits;     // row splits per tensor: the cluster has twice as many CTAs
    bool app_tuned;   // lagkv_plan_tune() fixed the uniform append shape: no pair kernel
    std::atomic<unsigned long long> attend_ready{0};  // attention kernels whose shared memory limit is raised
    std::atomic<unsigned long long> quant_ready{0}, write_ready{0};  // the same for caches in 8 bits with scales
    std::atomic<int> quant_clusters[64][3] = {};  // 1 + clusters of each size that fit the GPU at once; 0: not asked yet
    // lagkv_compress_prefill_host(): three streams and the events between them, made on first use
    std::mutex host_mu;
    bool host_ready = false;
    cudaStream_t host_stream[3] = {nullptr, nullptr, nullptr};  // copy in, compute, copy out
    cudaEvent_t host_start = nullptr, host_in[2] = {nullptr, nullptr}, host_comp[2] = {nullptr, nullptr},
                host_out[2] = {nullptr, nullptr};
    ~lagkv_plan_s() {
        if (!host_stream[0] && !host_start) return;
        int prev = -1;
        const bool sw = cfg.device >= 0 && cudaGetDevice(&prev) == cudaSuccess && prev != cfg.device &&
                        cudaSetDevice(cfg.device) == cudaSuccess;
        for (int i = 0; i < 3; ++i)
            if (host_stream[i]) cudaStreamDestroy(host_stream[i]);
        if (host_start) cudaEventDestroy(host_start);
        for (int i = 0; i < 2; ++i) {
            if (host_in[i]) cudaEventDestroy(host_in[i]);
            if (host_comp[i]) cudaEventDestroy(host_comp[i]);
            if (host_out[i]) cudaEventDestroy(host_out[i]);
        }
        if (sw) cudaSetDevice(prev);
    }
};

struct DeviceGuard {
    int prev = -1;
    bool switched = false;
    explicit DeviceGuard(int dev) {
        if (dev >= 0 && cudaGetDevice(&prev) == cudaSuccess && prev != dev)
            switched = (cudaSetDevice(dev) == cudaSuccess);
    }
    ~DeviceGuard() {
        if (switched) cudaSetDevice(prev);
    }
};

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The dynamic shared memory limit belongs to the function, not to the plan: only ever raise it, so
// that shapes of the same kernel with larger needs (this plan's or another's) keep launching.
inline bool raise_smem_limit(const void* fn, size_t smem) {
    static std::mutex limit_mu;  // read-then-raise must not interleave between threads
    std::lock_guard<std::mutex> lock(limit_mu);
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, fn) != cudaSuccess) return false;
    return size_t(attr.maxDynamicSharedSizeBytes) >= smem ||
           cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)) == cudaSuccess;
}

struct Strides {
    long long sb, sh, ss;
    // paged caches: block table and page geometry (block_table == nullptr: not paged)
    const int32_t* block_table = nullptr;
    long long page_stride = 0;
    int max_blocks = 0, page_shift = 0;
};
// Checks a paged layout and turns it into strides; S is the number of rows the call addresses.
inline int resolve_paged(const lagkv_config& c, const lagkv_paged_layout* lay, int64_t S, Strides* out) {
    if (lay == nullptr || lay->block_table == nullptr || (reinterpret_cast<uintptr_t>(lay->block_table) & 3u))
        return LAGKV_EINVAL;
    if (c.stride_b != 0 || c.stride_h != 0 || c.stride_s != 0) return LAGKV_EINVAL;  // the layout carries the strides
    const int ps = lay->page_size;
    if (ps < 16 || ps > (1 << 20) || (ps & (ps - 1)) != 0 || lay->max_blocks < 1) return LAGKV_EINVAL;
    if ((long long)lay->max_blocks * ps < S) return LAGKV_EINVAL;
    long long ss = lay->stride_s ? lay->stride_s : c.D;
    long long sh = lay->stride_h ? lay->stride_h : (long long)ps * ss;
    long long sp = lay->stride_page ? lay->stride_page : (long long)c.H_kv * sh;
    const int eb = elem_bytes(c.dtype), q = 16 / eb;  // strides are given in elements: multiples of 16 bytes
    if (ss < c.D || (ss % q) || (sh % q) || (sp % q) || sh < 0 || sp <= 0) return LAGKV_EINVAL;
    out->sb = 0;  // the kernels count in 16-bit units
    out->sh = sh * eb / 2;
    out->ss = ss * eb / 2;
    out->block_table = lay->block_table;
    out->page_stride = sp * eb / 2;
    out->max_blocks = lay->max_blocks;
    out->page_shift = 0;
    while ((1 << out->page_shift) < ps) ++out->page_shift;
    return LAGKV_OK;
}
inline int resolve_strides(const lagkv_config& c, int64_t S, Strides* out) {
    long long ss = c.stride_s ? c.stride_s : c.D;
    long long sh = c.stride_h ? c.stride_h : (long long)S * ss;
    long long sb = c.stride_b ? c.stride_b : (long long)c.H_kv * sh;
    const int eb = elem_bytes(c.dtype), q = 16 / eb;  // strides are given in elements: multiples of 16 bytes
    if (ss < c.D || (ss % q) || (sh % q) || (sb % q) || sh < 0 || sb < 0) return LAGKV_EINVAL;
    out->sb = sb * eb / 2;  // the kernels count in 16-bit units
    out->sh = sh * eb / 2;
    out->ss = ss * eb / 2;
    return LAGKV_OK;
}

inline int check_launch() {
    return cudaPeekAtLastError() == cudaSuccess ? LAGKV_OK : LAGKV_ECUDA;
}

// A launch that may begin while the one before it in the stream is ending: both kernels call griddepcontrol.
inline int launch_behind(const void* fn, unsigned grid, unsigned threads, void** args, size_t smem, cudaStream_t stream) {
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelExC(&cfg, fn, args) == cudaSuccess ? LAGKV_OK : LAGKV_ECUDA;
}
