// Attention over the cache -- host side of the C ABI: argument checks, workspace layout, launches.
#include "lagkv.h"

#include <cmath>
#include <cstring>
#include <cuda.h>
#include <limits>

#include "lagkv_attend_tables.h"
#include "lagkv_block_kernels.cuh"
#include "lagkv_plan.h"
#include "lagkv_tree_kernels.cuh"

using namespace lagkv;

namespace {

const AttendEntry* find_attend(int D, int dtype, int rows_wanted, bool blocks, int* index) {
    const AttendEntry* t;
    const int n = dtype == LAGKV_DTYPE_BF16   ? attend_bf16_kernels(&t)
                  : dtype == LAGKV_DTYPE_FP16 ? attend_fp16_kernels(&t)
                                              : attend_fp8_kernels(&t);
    // The smallest unit that holds all query rows, else the largest there is: rows of K and V are then read once.
    // In us, at 8 KV heads of 128 channels and 8192 rows of 16 sequences, for the units of 16, 32, 128 and 256 rows:
    //                           bf16                    fp8
    //     16 query rows        101  107   97  146        71   99  136  179
    //     32                   178  111   98  146       122  102  131  176
    //     64                   353  203  101  155       225  181  130  175
    //    128                   672  429  112  171       429  341  136  181
    // rows_of_unit() below asks for other units where the cache is small or large.
    const AttendEntry* best = nullptr;
    for (int i = 0; i < n; ++i) {
        if (t[i].D != D || (blocks && t[i].wide)) continue;
        const bool fits = t[i].rows >= rows_wanted, best_fits = best && best->rows >= rows_wanted;
        if (best == nullptr || (fits && (!best_fits || t[i].rows < best->rows)) || (!fits && !best_fits && t[i].rows > best->rows)) {
            best = t + i;
            *index = i;
        }
    }
    return best;
}

// Workspace: [status block | partials | who shares which unit | block choice].  Only the status block outlasts
// a call.
constexpr size_t kHead = kStatusWords * sizeof(int32_t);
size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

size_t partial_bytes(const lagkv_plan_s* plan, const AttendEntry& e) {
    return up256(size_t(plan->sm_count) * e.ctas_per_sm * 2 * e.partial_words * sizeof(float));
}
long long attend_units(const lagkv_plan_s* plan, const AttendEntry& e, int query_rows, int tokens) {
    return (long long)plan->cfg.B * plan->cfg.H_kv * tokens * ((query_rows + e.rows - 1) / e.rows);
}
// T tokens of G query heads per KV head are well formed
bool query_shape_ok(const lagkv_config& c, int T, int H_q) {
    return T >= 1 && T <= 64 && H_q >= c.H_kv && H_q % c.H_kv == 0 && H_q / c.H_kv <= 64;
}
// The choice of blocks: [chosen | 64-bit scores | 32-bit scores | how far these can be off]
struct ChoiceLayout {
    size_t keys, approx, error, total;
    ChoiceLayout(const lagkv_config& c, int T, int64_t blocks, int keep) {
        const size_t units = size_t(c.B) * T * c.H_kv;
        keys = up256(units * size_t(keep) * sizeof(int32_t));
        approx = keys + up256(units * size_t(blocks) * sizeof(unsigned long long));
        error = approx + up256(units * size_t(blocks) * sizeof(float));
        total = error + up256(units * (size_t(blocks) / kScoreChunk + 1) * sizeof(float));
    }
};
size_t choice_bytes(const lagkv_config& c, int T, int64_t blocks, int keep) {
    return blocks == 0 ? 0 : ChoiceLayout(c, T, blocks, keep).total;
}

template <int DT>
const void* score_kernel(int D) {
    return D == 64    ? reinterpret_cast<const void*>(&lagkv_block_score_kernel<DT, 64>)
           : D == 96  ? reinterpret_cast<const void*>(&lagkv_block_score_kernel<DT, 96>)
           : D == 128 ? reinterpret_cast<const void*>(&lagkv_block_score_kernel<DT, 128>)
                      : reinterpret_cast<const void*>(&lagkv_block_score_kernel<DT, 256>);
}

int fill_query(const lagkv_plan_s* plan, const lagkv_query* q, const void* Q, void* out, float* lse, AttendParams* P) {
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

constexpr int kMaxKeep = 4096, kMaxBlocks = 24576;  // the choice holds a unit's keys in shared memory

// The cache of a call: contiguous (layout == nullptr) or paged.
int fill_cache(const lagkv_plan_s* plan, const void* K, const void* V, int64_t S_cap, const lagkv_paged_layout* layout,
               int64_t num_pages, AttendParams* P) {
    const lagkv_config& c = plan->cfg;
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

int workspace_ok(const void* workspace, size_t bytes, size_t need) {
    if (workspace == nullptr || bytes < need) return LAGKV_EWORKSPACE;
    return (reinterpret_cast<uintptr_t>(workspace) & 255u) ? LAGKV_EINVAL : LAGKV_OK;
}

// The query rows that find_attend() is asked for.
// Small caches: units of 16 rows start faster and more CTAs take part; reading K and V for each of them costs little out of
// L2.  They win up to about 4 tiles per CTA (16-bit) or 12 (fp8, where wide tiles have to be widened).  8 KV heads of 128
// channels, units of 16 rows against the ones that hold all: bf16, 64 query rows, 256 / 1024 / 4096 rows 12.5 / 16 / 23
// against 15 / 17.5 / 22 us, 256 query rows 16 / 24 against 17.5 / 19; fp8, 64 query rows 12 / 14 / 20.5 against 18.5 / 21 / 26.
// Large 16-bit caches: 17 to 32 query rows go to the wide kernel as well: 20 and 32 query rows over 16 x 8 x 8192 rows
// of 128 channels 98 and 98 us against 107 and 111, over 4 x 8 x 8192 41 and 40 against 41 and 42, over 1 x 8 x 8192 26
// against 25; 20 and 32 over 16 x 8 x 8192 rows of 96 channels 86 and 87 against 91 and 94, 20 over 64 channels in pages
// 68 against 74.
int rows_of_unit(const lagkv_plan_s* plan, int query_rows, bool blocks, long long S_cap) {
    const lagkv_config& c = plan->cfg;
    const bool fp8 = c.dtype == LAGKV_DTYPE_FP8_E4M3;
    const long long heads = (long long)c.B * c.H_kv;
    if (blocks || query_rows <= 16) return query_rows;
    if (heads * ((query_rows + 15) / 16) * (S_cap / kAttendTile + kAttendLead) <= (long long)plan->sm_count * (fp8 ? 24 : 9)) return 16;
    return query_rows <= 32 && !fp8 && heads * S_cap >= 1 << 19 ? 33 : query_rows;
}

// Picks the kernel, finds room in the workspace and launches.  `extra`: bytes of the workspace behind
// the partials that the call uses itself.
int attend_prepare(lagkv_plan_t plan, int query_rows, int tokens, bool blocks, size_t extra, void* workspace, size_t bytes,
                   AttendParams* P, const AttendEntry** entry, unsigned char** rest) {
    int index = 0;
    const AttendEntry* e = find_attend(plan->cfg.D, plan->cfg.dtype, rows_of_unit(plan, query_rows, blocks, P->S_cap), blocks, &index);
    if (e == nullptr) return LAGKV_EUNSUPPORTED;
    const long long units = attend_units(plan, *e, query_rows, tokens);
    int rc = workspace_ok(workspace, bytes, kHead + 4096);
    if (rc != LAGKV_OK) return rc;
    const size_t pb = partial_bytes(plan, *e), sb = up256(size_t(units) * sizeof(int2));
    if (units * e->rows > 0x7fffffffll) return LAGKV_EINVAL;
    if (kHead + pb + sb + extra > bytes) return LAGKV_EWORKSPACE;
    unsigned char* base = static_cast<unsigned char*>(workspace);
    P->status = reinterpret_cast<int32_t*>(base);
    P->partials = reinterpret_cast<float*>(base + kHead);
    P->shared = reinterpret_cast<int2*>(base + kHead + pb);
    P->mtiles = (query_rows + e->rows - 1) / e->rows;
    P->ctas = plan->sm_count * e->ctas_per_sm;
    // (see attend_share) by the capacity, which may be far above the lengths: no more than 4.  One KV head of 20000 rows under
    // 32 tokens of 4 heads in 34 us, 45 with shares of one tile; of 8192 in 8 units 29 and 33.
    P->least = int(std::ceil(std::sqrt((P->S_cap / double(kWideTile) + kWideLead) / 6.0)));
    if (P->least > 4) P->least = 4;
    P->per_units = 1.f / (16.f * float(units));
    P->lead = e->wide ? kWideLead : kAttendLead;
    *entry = e;
    *rest = base + kHead + pb + sb;
    if (!(plan->attend_ready.load(std::memory_order_acquire) >> index & 1)) {
        if (!raise_smem_limit(e->fn, e->smem)) return LAGKV_ECUDA;
        plan->attend_ready.fetch_or(1ull << index, std::memory_order_release);
    }
    return LAGKV_OK;
}
typedef CUresult (*encode_tiled_t)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
encode_tiled_t encode_tiled() {
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
int cache_map(const lagkv_config& c, const AttendParams& P, const uint8_t* base, CUtensorMap* map) {
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
int launch_join(const AttendEntry& e, AttendParams& P, int query_rows, long long units, cudaStream_t stream) {
    const int rows = e.rows < query_rows ? e.rows : query_rows;
    void* args[] = {&P};
    return launch_behind(e.join, unsigned(units * ((rows + e.join_rows - 1) / e.join_rows)), e.join_threads, args, 0, stream);
}

int attend_launch(lagkv_plan_t plan, const AttendEntry& e, AttendParams& P, cudaStream_t stream) {
    CUtensorMap map_k, map_v;
    if (e.wide) {
        int rc = cache_map(plan->cfg, P, P.K, &map_k);
        if (rc == LAGKV_OK) rc = cache_map(plan->cfg, P, P.V, &map_v);
        if (rc != LAGKV_OK) return rc;
    }
    void* args[] = {&P, &map_k, &map_v};
    if (cudaLaunchKernel(e.fn, dim3((unsigned)P.ctas), dim3(e.threads), args, e.smem, stream) !=
        cudaSuccess)
        return LAGKV_ECUDA;
    const int rc = launch_join(e, P, P.T * P.G, (long long)P.B * P.H * P.mtiles, stream);
    if (rc != LAGKV_OK) return rc;
    return check_launch();
}

int attend_tree(lagkv_plan_t plan, const lagkv_query* query, const void* Q, const void* K, const void* V, int64_t S_cap,
                const lagkv_paged_layout* layout, int64_t num_pages, const int32_t* seq_len, const int32_t* draft_len,
                const uint64_t* tree_mask, void* out, float* lse, void* workspace, size_t bytes, void* cuda_stream) {
    if (plan == nullptr || seq_len == nullptr || V == nullptr) return LAGKV_EINVAL;
    AttendParams P;
    int rc = fill_query(plan, query, Q, out, lse, &P);
    if (rc == LAGKV_OK) rc = fill_cache(plan, K, V, S_cap, layout, num_pages, &P);
    if (rc != LAGKV_OK) return rc;
    if ((reinterpret_cast<uintptr_t>(seq_len) & 3u) || (reinterpret_cast<uintptr_t>(draft_len) & 3u) ||
        (reinterpret_cast<uintptr_t>(tree_mask) & 7u))
        return LAGKV_EINVAL;
    P.seq_len = seq_len;
    P.draft_len = draft_len;
    P.mask = reinterpret_cast<const unsigned long long*>(tree_mask);
    DeviceGuard guard(plan->cfg.device);
    const AttendEntry* e;
    unsigned char* rest;
    rc = attend_prepare(plan, P.T * P.G, 1, false, 0, workspace, bytes, &P, &e, &rest);
    if (rc != LAGKV_OK) return rc;
    return attend_launch(plan, *e, P, static_cast<cudaStream_t>(cuda_stream));
}

int tree_commit(lagkv_plan_t plan, void* K, void* V, int64_t S_cap, const lagkv_paged_layout* layout, int64_t num_pages,
                int32_t* seq_len, const int32_t* draft_len, int32_t T, const int32_t* accepted, const int32_t* n_accepted,
                void* workspace, size_t bytes, void* cuda_stream) {
    if (plan == nullptr || plan->cfg.device < 0 || seq_len == nullptr || accepted == nullptr || n_accepted == nullptr ||
        T < 1 || T > 64 || V == nullptr || K == V)
        return LAGKV_EINVAL;
    AttendParams P;
    std::memset(&P, 0, sizeof P);
    int rc = fill_cache(plan, K, V, S_cap, layout, num_pages, &P);
    if (rc == LAGKV_OK) rc = workspace_ok(workspace, bytes, kHead);
    if (rc != LAGKV_OK) return rc;
    if ((reinterpret_cast<uintptr_t>(seq_len) & 3u) || (reinterpret_cast<uintptr_t>(draft_len) & 3u) ||
        (reinterpret_cast<uintptr_t>(accepted) & 3u) || (reinterpret_cast<uintptr_t>(n_accepted) & 3u))
        return LAGKV_EINVAL;
    P.draft_len = draft_len;
    P.status = static_cast<int32_t*>(workspace);
    P.B = plan->cfg.B;
    P.H = plan->cfg.H_kv;
    P.T = T;
    DeviceGuard guard(plan->cfg.device);
    lagkv_tree_commit_kernel<<<plan->cfg.B, kCommitThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        P, static_cast<uint8_t*>(K), static_cast<uint8_t*>(V), int(row_bytes(plan->cfg) / 16), seq_len, accepted, n_accepted);
    return check_launch();
}

int block_shift_of(int rows) { return rows == 16 ? 4 : rows == 32 ? 5 : rows == 64 ? 6 : rows == 128 ? 7 : -1; }

int block_bounds(lagkv_plan_t plan, const void* K, int64_t S_cap, const lagkv_paged_layout* layout, int64_t num_pages,
                 const int32_t* from_len, const int32_t* seq_len, int32_t block_rows, void* bounds, int64_t blocks,
                 void* workspace, size_t bytes, void* cuda_stream) {
    if (plan == nullptr || plan->cfg.device < 0 || seq_len == nullptr || bounds == nullptr || !aligned16(bounds))
        return LAGKV_EINVAL;
    const lagkv_config& c = plan->cfg;
    AttendParams P;
    std::memset(&P, 0, sizeof P);
    int rc = fill_cache(plan, K, nullptr, S_cap, layout, num_pages, &P);
    if (rc == LAGKV_OK) rc = workspace_ok(workspace, bytes, kHead);
    if (rc != LAGKV_OK) return rc;
    P.block_shift = block_shift_of(block_rows);
    if (P.block_shift < 0 || blocks < 1 || (blocks << P.block_shift) < P.S_cap || K == bounds) return LAGKV_EINVAL;
    if ((reinterpret_cast<uintptr_t>(seq_len) & 3u) || (reinterpret_cast<uintptr_t>(from_len) & 3u)) return LAGKV_EINVAL;
    P.seq_len = seq_len;
    P.status = static_cast<int32_t*>(workspace);
    P.B = c.B;
    P.H = c.H_kv;
    DeviceGuard guard(c.device);
    // CTAs per (sequence, KV head): many for a whole cache, so that ragged lengths even out, few when only
    // the last rows have changed (each CTA's eight warps walk the blocks in strides either way)
    const long long units = (long long)c.B * c.H_kv, want = (long long)plan->sm_count * (from_len ? 4 : 32);
    const long long most = ((long long)P.S_cap + (8ll << P.block_shift) - 1) / (8ll << P.block_shift);
    long long per = (want + units - 1) / units;
    if (per > most) per = most;
    if (units * per > 0x7fffffffll) return LAGKV_EINVAL;
    const int cpr = int(row_bytes(c) / 16);
    const dim3 grid((unsigned)(units * per));
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (c.dtype == LAGKV_DTYPE_BF16)
        lagkv_block_bounds_kernel<0><<<grid, kBoundsThreads, 0, stream>>>(P, from_len, static_cast<uint8_t*>(bounds), blocks, int(per), cpr);
    else if (c.dtype == LAGKV_DTYPE_FP16)
        lagkv_block_bounds_kernel<1><<<grid, kBoundsThreads, 0, stream>>>(P, from_len, static_cast<uint8_t*>(bounds), blocks, int(per), cpr);
    else
        lagkv_block_bounds_kernel<2><<<grid, kBoundsThreads, 0, stream>>>(P, from_len, static_cast<uint8_t*>(bounds), blocks, int(per), cpr);
    return check_launch();
}

int attend_blocks(lagkv_plan_t plan, const lagkv_query* query, const lagkv_block_choice* choice, const void* Q,
                  const void* K, const void* V, int64_t S_cap, const lagkv_paged_layout* layout, int64_t num_pages,
                  const int32_t* seq_len, const void* bounds, void* out, float* lse, int32_t* idx_out, void* workspace,
                  size_t bytes, void* cuda_stream) {
    if (plan == nullptr || seq_len == nullptr || V == nullptr || choice == nullptr || bounds == nullptr || !aligned16(bounds))
        return LAGKV_EINVAL;
    AttendParams P;
    int rc = fill_query(plan, query, Q, out, lse, &P);
    if (rc == LAGKV_OK) rc = fill_cache(plan, K, V, S_cap, layout, num_pages, &P);
    if (rc != LAGKV_OK) return rc;
    P.block_shift = block_shift_of(choice->block_rows);
    if (P.block_shift < 0 || choice->keep < 1 || choice->sink_blocks < 0 || choice->recent_blocks < 0 ||
        (int64_t)choice->sink_blocks + choice->recent_blocks > choice->keep || choice->blocks < 1)
        return LAGKV_EINVAL;
    if (choice->keep > kMaxKeep || choice->blocks > kMaxBlocks) return LAGKV_EUNSUPPORTED;
    if ((choice->blocks << P.block_shift) < P.S_cap) return LAGKV_EINVAL;
    if ((reinterpret_cast<uintptr_t>(seq_len) & 3u) || (reinterpret_cast<uintptr_t>(idx_out) & 3u)) return LAGKV_EINVAL;
    const lagkv_config& c = plan->cfg;
    P.seq_len = seq_len;
    P.keep = choice->keep;
    const long long units = (long long)P.B * P.T * P.H;
    // blocks per CTA of the score kernel: few for one user's latency, more where CTAs abound
    ScoreShape S;
    S.blocks = choice->blocks;
    const long long small = units * ((choice->blocks + kScoreChunk - 1) / kScoreChunk) / (8ll * plan->sm_count);
    S.chunk = kScoreChunk * int(small < 1 ? 1 : small > 8 ? 8 : small);
    S.chunks = int((choice->blocks + S.chunk - 1) / S.chunk);
    if (units * S.chunks > 0x7fffffffll) return LAGKV_EINVAL;
    DeviceGuard guard(c.device);
    const AttendEntry* e;
    unsigned char* rest;
    rc = attend_prepare(plan, P.G, P.T, true, choice_bytes(c, P.T, choice->blocks, choice->keep), workspace, bytes, &P, &e, &rest);
    if (rc != LAGKV_OK) return rc;
    const ChoiceLayout lay(c, P.T, choice->blocks, choice->keep);
    int32_t* idx = idx_out ? idx_out : reinterpret_cast<int32_t*>(rest);
    unsigned long long* keys = reinterpret_cast<unsigned long long*>(rest + lay.keys);
    S.approx = reinterpret_cast<float*>(rest + lay.approx);
    S.error = reinterpret_cast<float*>(rest + lay.error);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const uint8_t* bd = static_cast<const uint8_t*>(bounds);
    const bool bf16 = c.dtype == LAGKV_DTYPE_BF16, fp16 = c.dtype == LAGKV_DTYPE_FP16;
    const void* score = bf16 ? score_kernel<0>(c.D) : fp16 ? score_kernel<1>(c.D) : score_kernel<2>(c.D);
    const void* select = bf16   ? reinterpret_cast<const void*>(&lagkv_block_select_kernel<0>)
                         : fp16 ? reinterpret_cast<const void*>(&lagkv_block_select_kernel<1>)
                                : reinterpret_cast<const void*>(&lagkv_block_select_kernel<2>);
    const size_t select_smem = size_t(choice->blocks) * 8;  // a score and a number each
    constexpr unsigned long long kSelectReady = 1ull << 63;
    if (!(plan->attend_ready.load(std::memory_order_acquire) & kSelectReady)) {
        if (!raise_smem_limit(select, size_t(kMaxBlocks) * 8)) return LAGKV_ECUDA;
        plan->attend_ready.fetch_or(kSelectReady, std::memory_order_release);
    }
    {
        void* args[] = {&P, &bd, &S};
        if (cudaLaunchKernel(score, dim3((unsigned)(units * S.chunks)), dim3(kScoreThreads), args, 0, stream) != cudaSuccess) return LAGKV_ECUDA;
    }
    {
        int D = c.D, sink = choice->sink_blocks, recent = choice->recent_blocks;
        void* args[] = {&P, &bd, &S, &D, &keys, &sink, &recent, &idx};
        rc = launch_behind(select, unsigned(units), kSelectThreads, args, select_smem, stream);
        if (rc != LAGKV_OK) return rc;
    }
    P.idx = idx;
    void* args[] = {&P};
    rc = launch_behind(e->fn, unsigned(P.ctas), unsigned(e->threads), args, e->smem, stream);
    if (rc == LAGKV_OK) rc = launch_join(*e, P, P.G, units * P.mtiles, stream);
    return rc == LAGKV_OK ? check_launch() : rc;
}

}  // namespace

extern "C" {

size_t lagkv_attend_workspace_bytes(lagkv_plan_t plan, int32_t T, int32_t H_q, int64_t blocks, int32_t keep) {
    if (plan == nullptr || !query_shape_ok(plan->cfg, T, H_q) || blocks < 0 || keep < 0) return 0;
    if (blocks > 0 && (keep < 1 || keep > kMaxKeep || blocks > kMaxBlocks)) return 0;
    const int G = H_q / plan->cfg.H_kv;
    // every smaller call of either kind: one token per unit with few query rows, all rows in one unit
    size_t partials = 0, units = 0;
    for (int rows : {1, 17, 33, 129, T * G}) {
        if (rows > T * G && !(rows == 33 && T * G > 16)) continue;  // 33: see rows_of_unit
        for (bool chosen : {false, true}) {
            int index;
            const AttendEntry* e = find_attend(plan->cfg.D, plan->cfg.dtype, rows, chosen, &index);
            if (e == nullptr) return 0;
            const size_t need = partial_bytes(plan, *e);
            if (need > partials) partials = need;
        }
    }
    const size_t most = size_t(T) * ((G + 15) / 16);  // units per (sequence, KV head): no unit has fewer than 16 rows
    const size_t dense = (size_t(T) * G + 15) / 16;
    units = size_t(plan->cfg.B) * plan->cfg.H_kv * (most > dense ? most : dense);
    const size_t body = partials + up256(units * sizeof(int2)) + choice_bytes(plan->cfg, T, blocks, keep);
    return kHead + (body < 4096 ? 4096 : body);
}

int lagkv_attend_workspace_init(lagkv_plan_t plan, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (plan == nullptr || plan->cfg.device < 0) return LAGKV_EINVAL;
    const int rc = workspace_ok(workspace, workspace_bytes, kHead);
    if (rc != LAGKV_OK) return rc;
    DeviceGuard guard(plan->cfg.device);
    return cudaMemsetAsync(workspace, 0, kHead, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? LAGKV_OK
                                                                                                        : LAGKV_ECUDA;
}

int lagkv_attend_tree(lagkv_plan_t plan, const lagkv_query* query, const void* Q, const void* K, const void* V,
                      int64_t S_cap, const int32_t* seq_len, const int32_t* draft_len, const uint64_t* tree_mask,
                      void* out, float* lse_out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return attend_tree(plan, query, Q, K, V, S_cap, nullptr, 0, seq_len, draft_len, tree_mask, out, lse_out, workspace,
                       workspace_bytes, cuda_stream);
}

int lagkv_attend_tree_paged(lagkv_plan_t plan, const lagkv_query* query, const void* Q, const void* K_pool,
                            const void* V_pool, const lagkv_paged_layout* layout, int64_t num_pages,
                            const int32_t* seq_len, const int32_t* draft_len, const uint64_t* tree_mask, void* out,
                            float* lse_out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (layout == nullptr) return LAGKV_EINVAL;
    return attend_tree(plan, query, Q, K_pool, V_pool, 0, layout, num_pages, seq_len, draft_len, tree_mask, out, lse_out,
                       workspace, workspace_bytes, cuda_stream);
}

int lagkv_tree_commit(lagkv_plan_t plan, void* K_cache, void* V_cache, int64_t S_cap, int32_t* seq_len,
                      const int32_t* draft_len, int32_t T, const int32_t* accepted, const int32_t* n_accepted,
                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return tree_commit(plan, K_cache, V_cache, S_cap, nullptr, 0, seq_len, draft_len, T, accepted, n_accepted, workspace,
                       workspace_bytes, cuda_stream);
}

int lagkv_tree_commit_paged(lagkv_plan_t plan, void* K_pool, void* V_pool, const lagkv_paged_layout* layout,
                            int64_t num_pages, int32_t* seq_len, const int32_t* draft_len, int32_t T,
                            const int32_t* accepted, const int32_t* n_accepted, void* workspace,
                            size_t workspace_bytes, void* cuda_stream) {
    if (layout == nullptr) return LAGKV_EINVAL;
    return tree_commit(plan, K_pool, V_pool, 0, layout, num_pages, seq_len, draft_len, T, accepted, n_accepted, workspace,
                       workspace_bytes, cuda_stream);
}

int lagkv_block_bounds(lagkv_plan_t plan, const void* K, int64_t S_cap, const int32_t* from_len, const int32_t* seq_len,
                       int32_t block_rows, void* bounds, int64_t blocks, void* workspace, size_t workspace_bytes,
                       void* cuda_stream) {
    return block_bounds(plan, K, S_cap, nullptr, 0, from_len, seq_len, block_rows, bounds, blocks, workspace,
                        workspace_bytes, cuda_stream);
}

int lagkv_block_bounds_paged(lagkv_plan_t plan, const void* K_pool, const lagkv_paged_layout* layout, int64_t num_pages,
                             const int32_t* from_len, const int32_t* seq_len, int32_t block_rows, void* bounds,
                             int64_t blocks, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (layout == nullptr) return LAGKV_EINVAL;
    return block_bounds(plan, K_pool, 0, layout, num_pages, from_len, seq_len, block_rows, bounds, blocks, workspace,
                        workspace_bytes, cuda_stream);
}

int lagkv_attend_blocks(lagkv_plan_t plan, const lagkv_query* query, const lagkv_block_choice* choice, const void* Q,
                        const void* K, const void* V, int64_t S_cap, const int32_t* seq_len, const void* bounds,
                        void* out, float* lse_out, int32_t* idx_out, void* workspace, size_t workspace_bytes,
                        void* cuda_stream) {
    return attend_blocks(plan, query, choice, Q, K, V, S_cap, nullptr, 0, seq_len, bounds, out, lse_out, idx_out,
                         workspace, workspace_bytes, cuda_stream);
}

int lagkv_attend_blocks_paged(lagkv_plan_t plan, const lagkv_query* query, const lagkv_block_choice* choice,
                              const void* Q, const void* K_pool, const void* V_pool, const lagkv_paged_layout* layout,
                              int64_t num_pages, const int32_t* seq_len, const void* bounds, void* out, float* lse_out,
                              int32_t* idx_out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (layout == nullptr) return LAGKV_EINVAL;
    return attend_blocks(plan, query, choice, Q, K_pool, V_pool, 0, layout, num_pages, seq_len, bounds, out, lse_out,
                         idx_out, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
