// What the host sides of the attention entry points share: checks of queries, caches and workspaces.
#pragma once
#include "lagkv.h"

#include <cmath>
#include <cstring>
#include <cuda.h>
#include <limits>

#include "lagkv_attend_tables.h"
#include "lagkv_plan.h"

namespace lagkv {

constexpr size_t kHead = kStatusWords * sizeof(int32_t);
inline size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

// T tokens of G query heads per KV head are well formed
inline bool query_shape_ok(const lagkv_config& c, int T, int H_q) {
    return T >= 1 && T <= 64 && H_q >= c.H_kv && H_q % c.H_kv == 0 && H_q / c.H_kv <= 64;
}
inline int fill_query(const lagkv_plan_s* plan, const lagkv_query* q, const void* Q, void* out, float* lse, AttendParams* P) {
    const lagkv_config& c = plan->cfg;
    if (q == nullptr || Q == nullptr || out == nullptr || c.device < 0) return LAGKV_EINVAL;
    if (!query_shape_ok(c, q->T, q->H_q)) return LAGKV_EINVAL;
    if (!aligned16(Q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3u) || Q == out) return LAGKV_EINVAL;
    const double scale = q->scale == 0.0 ? 1.0 / std::sqrt(double(c.D)) : q->scale;
    const double ks = q->k_scale == 0.0 ? 1.0 : q->k_scale, vs = q->v_scale == 0.0 ? 1.0 : q->v_scale;
    // 0 would make NaN of the -infinity of hidden rows
    const float scale_log2 = std::fmax(float(scale * ks * 1.4426950408889634), std::numeric_limits<float>::denorm_min());
    if (!(scale > 0.0) || !(ks > 0.0) || !(vs > 0.0) || !std::isfinite(scale_log2) || !std::isfinite(float(vs))) return LAGKV_EINVAL;
    const int64_t sh = q->stride_h ? q->stride_h : c.D;
    const int64_t st = q->stride_t ? q->stride_t : (int64_t)q->H_q * sh;
    const int64_t sb = q->stride_b ? q->stride_b : (int64_t)q->T * st;
    if (sh < 0 || st < 0 || sb < 0 || sh % 8 || st % 8 || sb % 8) return LAGKV_EINVAL;
    std::memset(P, 0, sizeof *P);
    P->Q = static_cast<const uint16_t*>(Q);
    P->out = static_cast<uint16_t*>(out);
    P->lse = lse;
    P->q_sb = sb;
    P->q_st = st;
    P->q_sh = sh;
    P->B = c.B;
    P->H = c.H_kv;
    P->G = q->H_q / c.H_kv;
    P->T = q->T;
    P->scale_log2 = scale_log2;
    P->v_scale = float(vs);
    return LAGKV_OK;
}

// The cache of a call: contiguous (layout == nullptr) or paged.
inline int fill_cache(const lagkv_config& c, const void* K, const void* V, int64_t S_cap, const lagkv_paged_layout* layout,
               int64_t num_pages, AttendParams* P) {
    if (K == nullptr || !aligned16(K) || !aligned16(V)) return LAGKV_EINVAL;
    Strides st;
    if (layout != nullptr) {
        if (layout->page_size < 1 || layout->max_blocks < 1 || num_pages < 1) return LAGKV_EINVAL;
        S_cap = (int64_t)layout->max_blocks * layout->page_size;
    }
    if (S_cap < 1 || S_cap > 0x7fffffffll - 65536) return LAGKV_EINVAL;
    if (layout != nullptr) {
        if (resolve_paged(c, layout, S_cap, &st) != LAGKV_OK) return LAGKV_EINVAL;
    } else if (resolve_strides(c, S_cap, &st) != LAGKV_OK) {
        return LAGKV_EINVAL;
    }
    P->K = static_cast<const uint8_t*>(K);
    P->V = static_cast<const uint8_t*>(V);
    P->S_cap = int(S_cap);
    P->sb = st.sb * 2;
    P->sh = st.sh * 2;
    P->ss = st.ss * 2;
    P->page_stride = st.page_stride * 2;
    P->block_table = st.block_table;
    P->max_blocks = st.max_blocks;
    P->page_shift = st.page_shift;
    P->num_pages = num_pages;
    return LAGKV_OK;
}

inline int fill_cache(const lagkv_plan_s* plan, const void* K, const void* V, int64_t S_cap, const lagkv_paged_layout* layout,
               int64_t num_pages, AttendParams* P) {
    return fill_cache(plan->cfg, K, V, S_cap, layout, num_pages, P);
}

inline int workspace_ok(const void* workspace, size_t bytes, size_t need) {
    if (workspace == nullptr || bytes < need) return LAGKV_EWORKSPACE;
    return (reinterpret_cast<uintptr_t>(workspace) & 255u) ? LAGKV_EINVAL : LAGKV_OK;
}

inline int block_shift_of(int rows) { return rows == 16 ? 4 : rows == 32 ? 5 : rows == 64 ? 6 : rows == 128 ? 7 : -1; }

typedef CUresult (*encode_tiled_t)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline encode_tiled_t encode_tiled() {
    static const encode_tiled_t fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<encode_tiled_t>(p);
    }();
    return fn;
}
// Tensor map of one cache tensor for the wide kernel: (channels, rows, heads, sequences or pages), boxes of
// 64 channels in 128-byte swizzled rows (fp8: whole rows as they are) and of a tile's rows, or a page's if fewer.
inline int cache_map(const lagkv_config& c, const AttendParams& P, const uint8_t* base, CUtensorMap* map) {
    const bool fp8 = c.dtype == LAGKV_DTYPE_FP8_E4M3, paged = P.block_table != nullptr;
    const cuuint64_t rows = paged ? 1ull << P.page_shift : (cuuint64_t)P.S_cap;
    const cuuint64_t dims[4] = {(cuuint64_t)c.D, rows, (cuuint64_t)c.H_kv, paged ? (cuuint64_t)P.num_pages : (cuuint64_t)c.B};
    const cuuint64_t strides[3] = {(cuuint64_t)P.ss, (cuuint64_t)P.sh, (cuuint64_t)(paged ? P.page_stride : P.sb)};
    const cuuint32_t box[4] = {fp8 ? (cuuint32_t)c.D : 64u, (cuuint32_t)(paged && rows < kWideTile ? rows : kWideTile), 1u, 1u};
    const cuuint32_t ones[4] = {1u, 1u, 1u, 1u};
    const CUtensorMapDataType type = fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16;
    const encode_tiled_t encode = encode_tiled();
    if (encode == nullptr) return LAGKV_ECUDA;
    const CUresult r = encode(map, type, 4, const_cast<uint8_t*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              fp8 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? LAGKV_OK : LAGKV_EUNSUPPORTED;  // strides of 2^40 bytes and more
}

// Behind an attention kernel: the kernel that joins the units which several CTAs share.
inline int launch_join(const AttendEntry& e, void* P, int query_rows, long long units, cudaStream_t stream) {
    const int rows = e.rows < query_rows ? e.rows : query_rows;
    void* args[] = {P};
    return launch_behind(e.join, unsigned(units * ((rows + e.join_rows - 1) / e.join_rows)), e.join_threads, args, 0, stream);
}

}  // namespace lagkv
