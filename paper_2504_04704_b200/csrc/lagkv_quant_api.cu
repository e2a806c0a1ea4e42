// Caches in 8 bits with block scales -- host side of the C ABI: argument checks, workspace layout, launches.
#include "lagkv.h"

#include <cmath>
#include <cstring>
#include <cuda.h>

#include "lagkv_attend_host.h"
#include "lagkv_attend_quant_tables.h"
#include "lagkv_plan.h"
#include "lagkv_quant_kernels.cuh"
#include "lagkv_quant_rules.h"

using namespace lagkv;

namespace {

bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

// The cache of a call as the attention sees it: contiguous (layout == nullptr) or paged; codes count as the library's
// 8-bit elements.
int fill_quant_cache(const lagkv_plan_s* plan, const lagkv_quant_cache* q, int64_t S_cap, const lagkv_paged_layout* layout,
                     int64_t num_pages, AttendParams* P) {
    if (q == nullptr || q->V == nullptr || q->K == q->V || q->K_scale == nullptr || q->V_scale == nullptr || q->K_scale == q->V_scale)
        return LAGKV_EINVAL;
    if (misaligned4(q->K_scale) || misaligned4(q->V_scale)) return LAGKV_EINVAL;
    if (q->format != LAGKV_QUANT_INT8 && q->format != LAGKV_QUANT_E4M3) return LAGKV_EINVAL;
    if (plan->cfg.dtype == LAGKV_DTYPE_FP8_E4M3) return LAGKV_EUNSUPPORTED;
    lagkv_config c = plan->cfg;
    c.dtype = LAGKV_DTYPE_FP8_E4M3;
    c.stride_b = q->stride_b;
    c.stride_h = q->stride_h;
    c.stride_s = q->stride_s;
    if (c.stride_b < 0 || c.stride_h < 0 || c.stride_s < 0) return LAGKV_EINVAL;
    const int rc = fill_cache(c, q->K, q->V, S_cap, layout, num_pages, P);
    if (rc != LAGKV_OK) return rc;
    P->block_shift = block_shift_of(q->block_rows);
    if (P->block_shift < 0 || q->blocks < 1 || q->blocks < (((int64_t)P->S_cap - 1) >> P->block_shift) + 1) return LAGKV_EINVAL;
    // a block lies in one page: a page that two sequences share then holds whole blocks
    if (layout != nullptr && q->block_rows > layout->page_size) return LAGKV_EINVAL;
    return LAGKV_OK;
}

// What writing and reading back share: cache, lengths, the 16-bit side's strides (0 = dense [B, H_kv, T, D]).
int fill_quant(const lagkv_plan_s* plan, const lagkv_quant_cache* q, int64_t S_cap, const lagkv_paged_layout* layout, int64_t num_pages,
               const int32_t* from_len, const int32_t* seq_len, int64_t T, int64_t stride_b, int64_t stride_h, int64_t stride_t,
               void* workspace, size_t bytes, QuantParams* P) {
    if (plan == nullptr || plan->cfg.device < 0 || seq_len == nullptr) return LAGKV_EINVAL;
    const lagkv_config& c = plan->cfg;
    AttendParams A;
    std::memset(&A, 0, sizeof A);
    int rc = fill_quant_cache(plan, q, S_cap, layout, num_pages, &A);
    if (rc == LAGKV_OK) rc = workspace_ok(workspace, bytes, kHead);
    if (rc != LAGKV_OK) return rc;
    if (misaligned4(seq_len) || misaligned4(from_len)) return LAGKV_EINVAL;
    if (T < 1 || T > 0x7fffffffll - 65536) return LAGKV_EINVAL;
    const int64_t st = stride_t ? stride_t : c.D, sh = stride_h ? stride_h : T * st, sb = stride_b ? stride_b : c.H_kv * sh;
    if (st < c.D || sh < 0 || sb < 0 || st % 8 || sh % 8 || sb % 8) return LAGKV_EINVAL;
    std::memset(P, 0, sizeof *P);
    P->codes[0] = static_cast<uint8_t*>(q->K);
    P->codes[1] = static_cast<uint8_t*>(q->V);
    P->scale[0] = q->K_scale;
    P->scale[1] = q->V_scale;
    P->sb = A.sb;
    P->sh = A.sh;
    P->ss = A.ss;
    P->page_stride = A.page_stride;
    P->block_table = A.block_table;
    P->num_pages = num_pages;
    P->blocks = q->blocks;
    P->B = c.B;
    P->H = c.H_kv;
    P->D = c.D;
    P->S_cap = A.S_cap;
    P->max_blocks = A.max_blocks;
    P->page_shift = A.page_shift;
    P->block_shift = A.block_shift;
    P->from_len = from_len;
    P->seq_len = seq_len;
    P->status = static_cast<int32_t*>(workspace);
    P->T = int(T);
    P->r_sb = sb;
    P->r_sh = sh;
    P->r_st = st;
    return LAGKV_OK;
}

struct WriteKernel {
    const void* fn;
    size_t smem;
};
template <int DT, int FORM, int GT>
WriteKernel write_kernel() { return {reinterpret_cast<const void*>(&lagkv_quant_write_kernel<DT, FORM, GT>), size_t(QuantWriteGeo<GT>::SMEM)}; }
template <int DT, int FORM>
WriteKernel write_kernel(int threads) {
    return threads == 32    ? write_kernel<DT, FORM, 32>()
           : threads == 64  ? write_kernel<DT, FORM, 64>()
           : threads == 128 ? write_kernel<DT, FORM, 128>()
           : threads == 256 ? write_kernel<DT, FORM, 256>()
                            : write_kernel<DT, FORM, 512>();
}

int quant_write(lagkv_plan_t plan, const lagkv_quant_cache* cache, int64_t S_cap, const lagkv_paged_layout* layout, int64_t num_pages,
                const lagkv_quant_source* source, const void* K, const void* V, const int32_t* from_len, const int32_t* seq_len,
                void* workspace, size_t bytes, void* cuda_stream) {
    if (source == nullptr || K == nullptr || V == nullptr || !aligned16(K) || !aligned16(V)) return LAGKV_EINVAL;
    QuantParams P;
    const int rc = fill_quant(plan, cache, S_cap, layout, num_pages, from_len, seq_len, source->T, source->stride_b, source->stride_h,
                              source->stride_t, workspace, bytes, &P);
    if (rc != LAGKV_OK) return rc;
    const lagkv_config& c = plan->cfg;
    P.rows[0] = static_cast<uint16_t*>(const_cast<void*>(K));
    P.rows[1] = static_cast<uint16_t*>(const_cast<void*>(V));
    if (K == cache->K || K == cache->V || V == cache->K || V == cache->V) return LAGKV_EINVAL;
    P.at_positions = source->at_positions != 0;
    P.n = source->T;
    if (source->take != nullptr) {
        if (misaligned4(source->take) || (source->take_heads != 1 && source->take_heads != c.H_kv) || source->take_rows < 1) return LAGKV_EINVAL;
        P.take = source->take;
        P.take_heads = source->take_heads;
        P.n = source->take_rows;
    }
    // the new rows of a block, at most, and the blocks that a sequence's may lie in
    const int R = cache->block_rows, rows = P.n < R ? P.n : R;
    long long most = P.n == 1 ? 1 : (P.n - 2) / R + 2;
    const long long all = ((long long)P.S_cap - 1) / R + 1;
    if (most > all) most = all;
    int threads = 32;
    while (threads / (c.D / 8) * kQuantPieces < rows) threads *= 2;
    const int groups = threads >= 256 ? 1 : 256 / threads;
    // groups per (sequence, head, tensor): 16 CTAs an SM even ragged lengths out
    const long long units = 2ll * c.B * c.H_kv, want = 16ll * plan->sm_count * groups;
    long long per = (want + units - 1) / units;
    if (per > most) per = most;
    if (units * per > 0x7fffffffll) return LAGKV_EINVAL;
    P.per = int(per);
    const bool bf16 = c.dtype == LAGKV_DTYPE_BF16, int8 = cache->format == LAGKV_QUANT_INT8;
    const WriteKernel w = bf16 ? (int8 ? write_kernel<0, FORM_INT8>(threads) : write_kernel<0, FORM_E4M3>(threads))
                               : (int8 ? write_kernel<1, FORM_INT8>(threads) : write_kernel<1, FORM_E4M3>(threads));
    DeviceGuard guard(c.device);
    const unsigned long long ready = 1ull << ((bf16 ? 0 : 8) + (int8 ? 0 : 16) + (threads >= 512 ? 4 : threads >> 6 > 2 ? 3 : threads >> 6));
    if (!(plan->write_ready.load(std::memory_order_acquire) & ready)) {
        if (!raise_smem_limit(w.fn, w.smem)) return LAGKV_ECUDA;
        plan->write_ready.fetch_or(ready, std::memory_order_release);
    }
    void* args[] = {&P};
    if (cudaLaunchKernel(w.fn, dim3(unsigned((units * per + groups - 1) / groups)), dim3(threads > 256 ? threads : 256), args, w.smem,
                         static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess)
        return LAGKV_ECUDA;
    return check_launch();
}

int quant_read(lagkv_plan_t plan, const lagkv_quant_cache* cache, int64_t S_cap, const lagkv_paged_layout* layout, int64_t num_pages,
               const int32_t* from_len, const int32_t* seq_len, const int32_t* idx, int64_t rows_out, void* K_out, void* V_out,
               void* workspace, size_t bytes, void* cuda_stream) {
    if (plan == nullptr || (K_out == nullptr && V_out == nullptr) || K_out == V_out || !aligned16(K_out) || !aligned16(V_out) || misaligned4(idx))
        return LAGKV_EINVAL;
    if (idx != nullptr && from_len != nullptr) return LAGKV_EINVAL;
    const lagkv_config& c = plan->cfg;
    QuantParams P;
    const int rc = fill_quant(plan, cache, S_cap, layout, num_pages, from_len, seq_len, rows_out, idx ? 0 : c.stride_b, idx ? 0 : c.stride_h,
                              idx ? 0 : c.stride_s, workspace, bytes, &P);
    if (rc != LAGKV_OK) return rc;
    for (const void* out : {K_out, V_out})
        if (out != nullptr && (out == cache->K || out == cache->V)) return LAGKV_EINVAL;
    P.rows[0] = static_cast<uint16_t*>(K_out);
    P.rows[1] = static_cast<uint16_t*>(V_out);
    P.take = idx;
    P.n = int(rows_out);
    // CTAs per (sequence, head, tensor): many for whole caches, so that ragged lengths even out; few behind from_len, where most
    // sequences of a decode step have a block to read (32 x 8 heads: 8 us against 18)
    const long long units = 2ll * c.B * c.H_kv, want = (from_len ? 8ll : 48ll) * plan->sm_count;
    const long long longest = idx ? rows_out : P.S_cap < rows_out ? P.S_cap : rows_out, rows = kReadThreads / (c.D / 8) * kReadPieces;
    long long per = (want + units - 1) / units;
    if (per > (longest + rows - 1) / rows) per = (longest + rows - 1) / rows;
    if (units * per > 0x7fffffffll) return LAGKV_EINVAL;
    P.per = int(per);
    const bool bf16 = c.dtype == LAGKV_DTYPE_BF16, int8 = cache->format == LAGKV_QUANT_INT8;
    const void* fn = bf16 ? (int8 ? reinterpret_cast<const void*>(&lagkv_quant_read_kernel<0, FORM_INT8>) : reinterpret_cast<const void*>(&lagkv_quant_read_kernel<0, FORM_E4M3>))
                          : (int8 ? reinterpret_cast<const void*>(&lagkv_quant_read_kernel<1, FORM_INT8>) : reinterpret_cast<const void*>(&lagkv_quant_read_kernel<1, FORM_E4M3>));
    DeviceGuard guard(c.device);
    void* args[] = {&P};
    if (cudaLaunchKernel(fn, dim3(unsigned(units * per)), dim3(kReadThreads), args, 0, static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess)
        return LAGKV_ECUDA;
    return check_launch();
}

// The kernel with units of `rows` query rows.
const AttendEntry* quant_entry(int D, int format, int rows, int* index) {
    const AttendEntry* t;
    const int n = format == LAGKV_QUANT_INT8 ? attend_int8_kernels(&t) : attend_e4m3_kernels(&t);
    for (int i = 0; i < n; ++i)
        if (t[i].D == D && t[i].rows == rows) {
            *index = i + (format == LAGKV_QUANT_INT8 ? 0 : 32);
            return t + i;
        }
    return nullptr;
}

// The kernel that a call takes.
const AttendEntry* find_quant(const lagkv_config& c, int format, int query_rows, int64_t S_cap, bool capped, int* index) {
    return quant_entry(c.D, format, quant_unit_rows((int64_t)c.B * c.H_kv, c.D, format == LAGKV_QUANT_INT8, query_rows, S_cap, capped), index);
}

// Workspace: [status block | partials | who shares which unit]
size_t partial_bytes(const lagkv_plan_s* plan, const AttendEntry& e) {
    return up256(size_t(plan->sm_count) * e.ctas_per_sm * 2 * e.partial_words * sizeof(float));
}
long long quant_units(const lagkv_config& c, const AttendEntry& e, int query_rows) {
    return (long long)c.B * c.H_kv * ((query_rows + e.rows - 1) / e.rows);
}

struct ClusterLaunch {
    cudaLaunchConfig_t config;
    cudaLaunchAttribute attr;
    ClusterLaunch(const AttendEntry& e, int ctas, long long units, cudaStream_t stream) {
        std::memset(&config, 0, sizeof config);
        config.gridDim = dim3(unsigned(units * ctas));
        config.blockDim = dim3(e.threads);
        config.dynamicSmemBytes = e.smem;
        config.stream = stream;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = unsigned(ctas);
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        config.attrs = &attr;
        config.numAttrs = 1;
    }
};
// CTAs of a unit's cluster, where a call takes that form (1: it does not).  How many of the size that the rule wants fit the GPU is
// asked once, which costs some microseconds; a size that the device refuses is no error.
int cluster_size(lagkv_plan_t plan, const AttendEntry& e, int index, long long units, int64_t S_cap) {
    if (e.cluster == nullptr) return 1;
    int fits[kClusterSizes];
    for (int i = 0; i < kClusterSizes; ++i) {
        const int known = plan->quant_clusters[index][i].load(std::memory_order_acquire);
        fits[i] = known == 0 ? 1 << 30 : known - 1;
    }
    for (;;) {
        const int ctas = quant_cluster_ctas(units, S_cap, fits);
        int i = 0;
        while (i < kClusterSizes && kClusterCtas[i] != ctas) ++i;
        if (i == kClusterSizes || fits[i] < 1 << 30) return ctas;
        const ClusterLaunch launch(e, ctas, 1, nullptr);
        int n = 0;
        if (!raise_smem_limit(e.cluster, e.smem) || cudaFuncSetAttribute(e.cluster, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, e.cluster, &launch.config) != cudaSuccess || n < 0) {
            n = 0;
            cudaGetLastError();
        }
        fits[i] = n;
        plan->quant_clusters[index][i].store(n + 1, std::memory_order_release);
    }
}

int attend_quant(lagkv_plan_t plan, const lagkv_query* query, double cap, const lagkv_quant_cache* cache, const void* Q, int64_t S_cap,
                 const lagkv_paged_layout* layout, int64_t num_pages, const int32_t* seq_len, const int32_t* draft_len,
                 const uint64_t* tree_mask, void* out, float* lse, void* workspace, size_t bytes, void* cuda_stream) {
    if (plan == nullptr || seq_len == nullptr) return LAGKV_EINVAL;
    QuantAttendParams P;
    std::memset(static_cast<void*>(&P), 0, sizeof P);
    int rc = fill_query(plan, query, Q, out, lse, &P);
    if (rc == LAGKV_OK) rc = fill_quant_cache(plan, cache, S_cap, layout, num_pages, &P);
    if (rc != LAGKV_OK) return rc;
    if (misaligned4(seq_len) || misaligned4(draft_len) || (reinterpret_cast<uintptr_t>(tree_mask) & 7u)) return LAGKV_EINVAL;
    if (!(cap >= 0.0) || (cap > 0.0 && (!std::isfinite(float(cap * 1.4426950408889634)) || !(float(cap) >= 0x1p-100f)))) return LAGKV_EINVAL;
    if (cap > 0.0) {
        P.cap_log2 = float(cap * 1.4426950408889634);
        P.cap_inv = float(1.0 / (cap * 1.4426950408889634));
    }
    P.K_scale = cache->K_scale;
    P.V_scale = cache->V_scale;
    P.blocks = cache->blocks;
    P.half = plan->cfg.dtype == LAGKV_DTYPE_FP16;
    P.seq_len = seq_len;
    P.draft_len = draft_len;
    P.mask = reinterpret_cast<const unsigned long long*>(tree_mask);
    const int query_rows = P.T * P.G;
    int index = 0;
    const AttendEntry* e = find_quant(plan->cfg, cache->format, query_rows, P.S_cap, cap > 0.0, &index);
    if (e == nullptr) return LAGKV_EUNSUPPORTED;
    const long long units = quant_units(plan->cfg, *e, query_rows);
    rc = workspace_ok(workspace, bytes, kHead);
    if (rc != LAGKV_OK) return rc;
    const size_t pb = partial_bytes(plan, *e), sb = up256(size_t(units) * sizeof(int2));
    if (units * e->rows > 0x7fffffffll) return LAGKV_EINVAL;
    if (kHead + pb + sb > bytes) return LAGKV_EWORKSPACE;
    unsigned char* base = static_cast<unsigned char*>(workspace);
    P.status = reinterpret_cast<int32_t*>(base);
    P.partials = reinterpret_cast<float*>(base + kHead);
    P.shared = reinterpret_cast<int2*>(base + kHead + pb);
    P.mtiles = (query_rows + e->rows - 1) / e->rows;
    P.ctas = plan->sm_count * e->ctas_per_sm;
    P.per_units = 1.f / (16.f * float(units));
    P.least = int(std::ceil(std::sqrt((P.S_cap / double(kWideTile) + kWideLead) / 6.0)));  // as for other caches
    if (P.least > 4) P.least = 4;
    P.lead = e->wide ? kWideLead : kAttendLead;
    DeviceGuard guard(plan->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int ctas = cluster_size(plan, *e, index, units, P.S_cap);
    if (ctas > 1) {
        const ClusterLaunch launch(*e, ctas, units, stream);
        void* cluster_args[] = {&P};
        if (cudaLaunchKernelExC(&launch.config, e->cluster, cluster_args) == cudaSuccess) return check_launch();
        cudaGetLastError();  // refused after all: the form without clusters serves the call
    }
    if (!(plan->quant_ready.load(std::memory_order_acquire) >> index & 1)) {
        if (!raise_smem_limit(e->fn, e->smem)) return LAGKV_ECUDA;
        plan->quant_ready.fetch_or(1ull << index, std::memory_order_release);
    }
    CUtensorMap map_k, map_v;
    if (e->wide) {
        lagkv_config codes = plan->cfg;
        codes.dtype = LAGKV_DTYPE_FP8_E4M3;
        rc = cache_map(codes, P, P.K, &map_k);
        if (rc == LAGKV_OK) rc = cache_map(codes, P, P.V, &map_v);
        if (rc != LAGKV_OK) return rc;
    }
    void* args[] = {&P, &map_k, &map_v};
    if (cudaLaunchKernel(e->fn, dim3((unsigned)P.ctas), dim3(e->threads), args, e->smem, stream) != cudaSuccess) return LAGKV_ECUDA;
    rc = launch_join(*e, &P, query_rows, units, stream);
    return rc == LAGKV_OK ? check_launch() : rc;
}

}  // namespace

extern "C" {

int lagkv_quant_write(lagkv_plan_t plan, const lagkv_quant_cache* cache, int64_t S_cap, const lagkv_quant_source* source, const void* K,
                      const void* V, const int32_t* from_len, const int32_t* seq_len, void* workspace, size_t workspace_bytes,
                      void* cuda_stream) {
    return quant_write(plan, cache, S_cap, nullptr, 0, source, K, V, from_len, seq_len, workspace, workspace_bytes, cuda_stream);
}

int lagkv_quant_write_paged(lagkv_plan_t plan, const lagkv_quant_cache* cache, const lagkv_paged_layout* layout, int64_t num_pages,
                            const lagkv_quant_source* source, const void* K, const void* V, const int32_t* from_len,
                            const int32_t* seq_len, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (layout == nullptr) return LAGKV_EINVAL;
    return quant_write(plan, cache, 0, layout, num_pages, source, K, V, from_len, seq_len, workspace, workspace_bytes, cuda_stream);
}

int lagkv_quant_read(lagkv_plan_t plan, const lagkv_quant_cache* cache, int64_t S_cap, const int32_t* from_len, const int32_t* seq_len,
                     const int32_t* idx, int64_t rows_out, void* K_out, void* V_out, void* workspace, size_t workspace_bytes,
                     void* cuda_stream) {
    return quant_read(plan, cache, S_cap, nullptr, 0, from_len, seq_len, idx, rows_out, K_out, V_out, workspace, workspace_bytes,
                      cuda_stream);
}

int lagkv_quant_read_paged(lagkv_plan_t plan, const lagkv_quant_cache* cache, const lagkv_paged_layout* layout, int64_t num_pages,
                           const int32_t* from_len, const int32_t* seq_len, const int32_t* idx, int64_t rows_out, void* K_out,
                           void* V_out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (layout == nullptr) return LAGKV_EINVAL;
    return quant_read(plan, cache, 0, layout, num_pages, from_len, seq_len, idx, rows_out, K_out, V_out, workspace, workspace_bytes,
                      cuda_stream);
}

size_t lagkv_attend_quant_workspace_bytes(lagkv_plan_t plan, int32_t T, int32_t H_q) {
    if (plan == nullptr || !query_shape_ok(plan->cfg, T, H_q)) return 0;
    // every smaller call, in either format, and whichever unit it takes
    size_t partials = 0;
    const int rows_all = T * (H_q / plan->cfg.H_kv);
    for (int format : {LAGKV_QUANT_INT8, LAGKV_QUANT_E4M3})
        for (int rows : {8, 16, 32, 128, 256}) {
            if (rows == 256 && rows_all <= 128) continue;
            int index;
            const AttendEntry* e = quant_entry(plan->cfg.D, format, rows, &index);
            if (e != nullptr && partial_bytes(plan, *e) > partials) partials = partial_bytes(plan, *e);
        }
    const size_t units = size_t(plan->cfg.B) * plan->cfg.H_kv * ((rows_all + 7) / 8);  // none has fewer rows
    return kHead + partials + up256(units * sizeof(int2));
}

int lagkv_attend_quant(lagkv_plan_t plan, const lagkv_query* query, double cap, const lagkv_quant_cache* cache, const void* Q,
                       int64_t S_cap, const int32_t* seq_len, const int32_t* draft_len, const uint64_t* tree_mask, void* out,
                       float* lse_out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return attend_quant(plan, query, cap, cache, Q, S_cap, nullptr, 0, seq_len, draft_len, tree_mask, out, lse_out, workspace,
                        workspace_bytes, cuda_stream);
}

int lagkv_attend_quant_paged(lagkv_plan_t plan, const lagkv_query* query, double cap, const lagkv_quant_cache* cache, const void* Q,
                             const lagkv_paged_layout* layout, int64_t num_pages, const int32_t* seq_len, const int32_t* draft_len,
                             const uint64_t* tree_mask, void* out, float* lse_out, void* workspace, size_t workspace_bytes,
                             void* cuda_stream) {
    if (layout == nullptr) return LAGKV_EINVAL;
    return attend_quant(plan, query, cap, cache, Q, 0, layout, num_pages, seq_len, draft_len, tree_mask, out, lse_out, workspace,
                        workspace_bytes, cuda_stream);
}

}  // extern "C"
