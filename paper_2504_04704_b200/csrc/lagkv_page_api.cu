// The pages of a paged cache -- host side of the C ABI: argument checks and launches.
#include "lagkv.h"

#include <cstring>

#include "lagkv_page_kernels.cuh"
#include "lagkv_plan.h"

using namespace lagkv;

namespace {

// Workspace: [status | arrival counter, 256 bytes | per-pair and per-sequence numbers or new names | lists]
constexpr size_t kFixedWords = 2 * kStatusWords;
size_t work_words(const lagkv_plan_s* plan, int64_t num_pages) {
    const size_t pairs = size_t(plan->cfg.B) * (kPairWords + 1) + 1, names = size_t(num_pages) + 1;
    return ((pairs > names ? pairs : names) + 63) & ~size_t(63);
}

int fill(const lagkv_plan_s* plan, const int32_t* table, int32_t max_blocks, int32_t page_size, int64_t num_pages, int32_t* refs,
         void* workspace, size_t bytes, PageParams* P) {
    if (plan == nullptr || plan->cfg.device < 0 || table == nullptr || refs == nullptr) return LAGKV_EINVAL;
    if (max_blocks < 1 || page_size < 16 || page_size > (1 << 20) || (page_size & (page_size - 1)) != 0) return LAGKV_EINVAL;
    if ((int64_t)max_blocks * page_size > 0x7fffffffll - 65536 || num_pages < 1 || num_pages > 0x3fffffffll) return LAGKV_EINVAL;
    if ((reinterpret_cast<uintptr_t>(table) & 3u) || (reinterpret_cast<uintptr_t>(refs) & 3u)) return LAGKV_EINVAL;
    if (workspace == nullptr || bytes < lagkv_pages_workspace_bytes(const_cast<lagkv_plan_s*>(plan), num_pages)) return LAGKV_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return LAGKV_EINVAL;
    std::memset(P, 0, sizeof *P);
    P->table = const_cast<int32_t*>(table);
    P->refs = refs;
    P->status = static_cast<int32_t*>(workspace);
    P->arrived = P->status + kStatusWords;
    P->work = P->status + kFixedWords;
    P->list = P->work + work_words(plan, num_pages);
    P->num_pages = num_pages;
    P->B = plan->cfg.B;
    P->H = plan->cfg.H_kv;
    P->max_blocks = max_blocks;
    while ((1 << P->page_shift) < page_size) ++P->page_shift;
    return LAGKV_OK;
}
int fill_pools(const lagkv_plan_s* plan, void* K, void* V, const lagkv_paged_layout* layout, PageParams* P) {
    const lagkv_config& c = plan->cfg;
    if (K == nullptr || V == nullptr || K == V || !aligned16(K) || !aligned16(V)) return LAGKV_EINVAL;
    Strides st;
    if (resolve_paged(c, layout, (int64_t)layout->max_blocks * layout->page_size, &st) != LAGKV_OK) return LAGKV_EINVAL;
    P->K = static_cast<uint8_t*>(K);
    P->V = static_cast<uint8_t*>(V);
    P->page_stride = st.page_stride * 2;
    P->sh = st.sh * 2;
    P->ss = st.ss * 2;
    P->vpr = int(row_bytes(c) / 16);
    const long long rb = (long long)row_bytes(c);
    P->dense = P->ss == rb && P->sh == rb << P->page_shift;
    if (((long long)P->H << P->page_shift) * P->vpr > 0x7fffffffll) return LAGKV_EUNSUPPORTED;
    return LAGKV_OK;
}
// enough CTAs for every SM to be full; the kernels walk their items in strides
int copy_grid(const lagkv_plan_s* plan) { return plan->sm_count * 8; }

}  // namespace

extern "C" {

size_t lagkv_pages_workspace_bytes(lagkv_plan_t plan, int64_t num_pages) {
    if (plan == nullptr || num_pages < 1 || num_pages > 0x3fffffffll) return 0;
    const size_t words = kFixedWords + work_words(plan, num_pages) + 2 * size_t(num_pages);
    return (words * sizeof(int32_t) + 255) & ~size_t(255);
}

int lagkv_pages_workspace_init(lagkv_plan_t plan, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (plan == nullptr || plan->cfg.device < 0) return LAGKV_EINVAL;
    if (workspace == nullptr || workspace_bytes < kFixedWords * sizeof(int32_t)) return LAGKV_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return LAGKV_EINVAL;
    DeviceGuard guard(plan->cfg.device);
    return cudaMemsetAsync(workspace, 0, kFixedWords * sizeof(int32_t), static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess
               ? LAGKV_OK
               : LAGKV_ECUDA;
}

int lagkv_pages_release(lagkv_plan_t plan, int32_t* block_table, int32_t max_blocks, int32_t page_size, int64_t num_pages,
                        int32_t* refs, const int32_t* keep_len, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    PageParams P;
    const int rc = fill(plan, block_table, max_blocks, page_size, num_pages, refs, workspace, workspace_bytes, &P);
    if (rc != LAGKV_OK) return rc;
    if (keep_len == nullptr || (reinterpret_cast<uintptr_t>(keep_len) & 3u)) return LAGKV_EINVAL;
    DeviceGuard guard(plan->cfg.device);
    const long long want = ((long long)P.B * max_blocks + kPageThreads - 1) / kPageThreads, most = (long long)plan->sm_count * 8;
    lagkv_pages_release_kernel<<<unsigned(want < most ? want : most), kPageThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        P, keep_len);
    return check_launch();
}

int lagkv_pages_reserve(lagkv_plan_t plan, int32_t* block_table, int32_t max_blocks, int32_t page_size, int64_t num_pages,
                        int32_t* refs, const int32_t* want_len, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    PageParams P;
    const int rc = fill(plan, block_table, max_blocks, page_size, num_pages, refs, workspace, workspace_bytes, &P);
    if (rc != LAGKV_OK) return rc;
    if (want_len == nullptr || (reinterpret_cast<uintptr_t>(want_len) & 3u)) return LAGKV_EINVAL;
    DeviceGuard guard(plan->cfg.device);
    lagkv_pages_reserve_kernel<<<P.B, kScanThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(P, want_len);
    return check_launch();
}

int lagkv_pages_fork(lagkv_plan_t plan, void* K_pool, void* V_pool, const lagkv_paged_layout* layout, int64_t num_pages,
                     int32_t* refs, int32_t* seq_len, int32_t* static_len, const int32_t* src, const int32_t* dst, int32_t n,
                     void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (layout == nullptr || plan == nullptr) return LAGKV_EINVAL;
    PageParams P;
    int rc = fill(plan, layout->block_table, layout->max_blocks, layout->page_size, num_pages, refs, workspace, workspace_bytes, &P);
    if (rc == LAGKV_OK) rc = fill_pools(plan, K_pool, V_pool, layout, &P);
    if (rc != LAGKV_OK) return rc;
    if (seq_len == nullptr || static_len == nullptr || src == nullptr || dst == nullptr || n < 0 || n > plan->cfg.B) return LAGKV_EINVAL;
    if ((reinterpret_cast<uintptr_t>(seq_len) & 3u) || (reinterpret_cast<uintptr_t>(static_len) & 3u) ||
        (reinterpret_cast<uintptr_t>(src) & 3u) || (reinterpret_cast<uintptr_t>(dst) & 3u))
        return LAGKV_EINVAL;
    if (n == 0) return LAGKV_OK;
    DeviceGuard guard(plan->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    lagkv_pages_fork_plan_kernel<<<n, kScanThreads, 0, stream>>>(P, seq_len, static_len, src, dst);
    void* args[] = {&P, &seq_len, &static_len, &src, &dst, &n};
    rc = launch_behind(reinterpret_cast<const void*>(&lagkv_pages_fork_kernel), unsigned(copy_grid(plan)), kPageThreads, args, 0, stream);
    return rc == LAGKV_OK ? check_launch() : rc;
}

int lagkv_pages_compact(lagkv_plan_t plan, void* K_pool, void* V_pool, const lagkv_paged_layout* layout, int64_t num_pages,
                        int32_t* refs, int32_t* live_out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (layout == nullptr || plan == nullptr) return LAGKV_EINVAL;
    PageParams P;
    int rc = fill(plan, layout->block_table, layout->max_blocks, layout->page_size, num_pages, refs, workspace, workspace_bytes, &P);
    if (rc == LAGKV_OK) rc = fill_pools(plan, K_pool, V_pool, layout, &P);
    if (rc != LAGKV_OK) return rc;
    if (live_out == nullptr || (reinterpret_cast<uintptr_t>(live_out) & 3u)) return LAGKV_EINVAL;
    DeviceGuard guard(plan->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    lagkv_pages_compact_plan_kernel<<<1, kScanThreads, 0, stream>>>(P, live_out);
    void* args[] = {&P};
    rc = launch_behind(reinterpret_cast<const void*>(&lagkv_pages_compact_kernel), unsigned(copy_grid(plan)), kPageThreads, args, 0, stream);
    return rc == LAGKV_OK ? check_launch() : rc;
}

}  // extern "C"
