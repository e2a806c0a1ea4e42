/*
 * lagkv.h -- C ABI of the B200 (sm_100a) LagKV KV-cache compression library.
 *
 * LagKV (arXiv 2504.04704, Section 2.2) shortens a transformer KV cache without looking
 * at attention weights.  After an attention-sink prefix of S rows the cache is cut into
 * partitions of L rows ("lag size").  Partition p is scored against partition p+1: the
 * per-channel min and max of the next partition (Eq. 7, Eq. 8) normalise the current one
 * (Eq. 9); the standard deviation over head_dim of every normalised token goes through a
 * softmax over the partition's tokens (Eq. 10), once for K and once for V, and the two are
 * added (Eq. 11).  Per head and per partition the k = ceil(r*L) best tokens are kept
 * (last bullet of Section 2.2); the last full partition plus the Mod(Ls-S, L) trailing
 * rows stay as a sliding window.  The resulting length is Eq. 12.
 *
 * Conventions shared by every entry point
 *   - All cache pointers are DEVICE pointers to data in the plan's storage format (bf16 by
 *     default, fp16 or fp8 e4m3 when the plan says so: "bf16" below stands for the plan's
 *     format), 16-byte aligned; scalars and the config struct are host values.  The library allocates no device memory and
 *     never synchronises the stream, except in lagkv_read_status().
 *   - A cache is addressed as  base + b*stride_b + h*stride_h + s*stride_s + d  (strides
 *     in elements, channel stride 1).  A stride given as 0 means "contiguous
 *     [B, H, S, D]" for the S passed to the call.  Strides must be multiples of 16 bytes
 *     (8 elements of a 16-bit format, 16 of fp8).
 *   - "Layers" have no separate dimension: fold them into B (one allocation
 *     [layers*B, H, S, D]) so that one call covers a whole model.
 *   - Every function returning int returns a lagkv_status code (0 = success).
 *     Errors detected on the host leave all buffers untouched.  Errors detected on the
 *     device (a bounded wait that ran out, an append that would overflow idx capacity)
 *     are recorded in the status block at the start of the workspace and reported by
 *     lagkv_read_status(); the kernels never trap or spin forever.  After LAGKV_ETIMEOUT
 *     the outputs of that call are incomplete: a prefill's K_out / V_out / idx_out hold
 *     undefined rows; an append leaves seq_len / static_len of every sequence one of whose
 *     heads gave up as they were before the call, and the rows of such a sequence behind
 *     its static part are undefined (other heads may already have been moved).  The
 *     workspace itself stays usable: the per-sequence counters return to zero.
 *   - The workspace is caller-owned device memory of at least lagkv_workspace_bytes()
 *     bytes, 256-byte aligned, cleared once with lagkv_workspace_init() and then reusable
 *     across calls on the same stream.  Calls sharing a workspace must not overlap.
 */
#ifndef LAGKV_H_
#define LAGKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lagkv_plan_s *lagkv_plan_t;

enum lagkv_status {
    LAGKV_OK = 0,
    LAGKV_EINVAL = 1,       /* null pointer, misalignment, bad shape / stride / size  */
    LAGKV_EUNSUPPORTED = 2, /* valid request the library has no kernel for            */
    LAGKV_EWORKSPACE = 3,   /* workspace missing or too small                         */
    LAGKV_ECUDA = 4,        /* CUDA runtime error at launch (left sticky, not cleared)*/
    LAGKV_ETIMEOUT = 5,     /* device: a bounded wait on an async copy ran out        */
    LAGKV_ECAPACITY = 6,    /* device: append needed more chunks than max_new_chunks  */
    LAGKV_ENOALLOC_LIMIT = 7 /* request larger than LAGKV_NOALLOC_SCRATCH_BYTES        */
};

enum lagkv_variant {
    LAGKV_VARIANT_LAGKV = 0,   /* Eq. 7-11: statistics from the next partition        */
    LAGKV_VARIANT_LOCALKV = 1, /* Eq. 14, Eq. 15: statistics from the partition itself */
    LAGKV_VARIANT_L2NORM = 2   /* Eq. 16: score = -||K row||_2, no softmax, V is only
                                  gathered.  Section 4.3 leaves the first two layers of
                                  the model uncompressed for this variant: layers have
                                  no dimension here, so the caller keeps those two
                                  layers out of the batch it folds into B               */
};

enum lagkv_dtype {
    LAGKV_DTYPE_BF16 = 0, /* the default (a zeroed field)                                */
    LAGKV_DTYPE_FP16 = 1, /* IEEE binary16 caches                                        */
    LAGKV_DTYPE_FP8_E4M3 = 2 /* one byte per element: 1 sign, 4 exponent (bias 7), 3 fraction
                             bits, no infinities, 0x7f / 0xff are NaN (the "e4m3fn" of the
                             deep-learning frameworks).  The paper names no storage format
                             and no scale; none is needed: whatever positive per-tensor,
                             per-head or per-channel scale the caller's quantiser uses, it
                             cancels in Eq. 9 (the same scale multiplies value, min and max),
                             so the scores are those of the stored bytes and the kept rows
                             are copied byte for byte.                                     */
};

typedef struct {
    int32_t B;          /* sequences (times layers when folded), >= 1                 */
    int32_t H_kv;       /* KV heads per sequence, >= 1; selection is per KV head      */
    int32_t D;          /* head_dim; supported: 64, 96, 128, 256 (128 is tuned)      */
    int32_t sink;       /* S: attention-sink rows kept verbatim, >= 0                 */
    int32_t lag;        /* L: partition size, 2 <= L <= 8192                          */
    double keep_ratio;  /* r in (0, 1]; k = ceil(r*L - 1e-9) clamped to [1, L]        */
    int32_t keep_k;     /* if > 0, k directly (overrides keep_ratio)                  */
    int32_t std_ddof;   /* divisor of the variance is D - std_ddof: 0 or 1            */
    int32_t variant;    /* enum lagkv_variant                                         */
    int64_t stride_b;   /* input-cache strides in elements; 0 = contiguous (see top)  */
    int64_t stride_h;
    int64_t stride_s;
    int32_t device;     /* CUDA device ordinal the plan launches on                   */
    int32_t dtype;      /* enum lagkv_dtype: storage format of every cache of the plan;
                           the paper names none, and the arithmetic after the exact
                           widening to fp32 is the same                               */
} lagkv_config;

/*
 * Build an immutable plan from a config (Section 2.2: S, L, r fix the whole pass).
 * Host work plus one-time CUDA attribute queries on cfg->device; no stream work.
 * On success *out owns host memory freed by lagkv_plan_destroy().
 */
int lagkv_plan(const lagkv_config *cfg, lagkv_plan_t *out);
void lagkv_plan_destroy(lagkv_plan_t plan);

/* k, the rows kept per compressed partition (r*L, text before Eq. 12). */
int32_t lagkv_keep_count(lagkv_plan_t plan);

/*
 * Eq. 12 generalised to a cache whose first static_len rows (sink + already compressed
 * part) are left alone:  static_len + k*(n-1) + L + rem  with n = floor(rest/L),
 * rem = rest mod L, rest = seq_len - static_len;  seq_len itself when rest < 2L (third
 * bullet of Section 2.2).  Pure host arithmetic.  static_len < 0 means "the plan's sink".
 */
int64_t lagkv_compressed_len(lagkv_plan_t plan, int64_t seq_len, int64_t static_len);

/*
 * The two lengths of a sequence after a pass (Section 2.2, bullets 2-4; Eq. 12): what
 * lagkv_compress_append() writes to seq_len[b] and static_len[b] on the device, computed on the
 * host so that a driver loop can mirror them without a read-back.  rest < 2L: both unchanged.
 * static_len < 0 means "the plan's sink".  Returns LAGKV_EINVAL for seq_len < static_len.
 */
int lagkv_lengths_after(lagkv_plan_t plan, int64_t seq_len, int64_t static_len, int64_t *new_seq_len,
                        int64_t *new_static_len);

/*
 * Inverse of Eq. 12 / Eq. 13 as used for the adaptive retention ratio of Section 3.2:
 * the smallest k in [1, L] whose compression ratio C = 1 - L_R/Ls does not exceed
 * target_C for a prompt of Ls rows.  Host arithmetic.  Returns k (L when no compression
 * is possible because Ls < S + 2L).
 */
int32_t lagkv_keep_for_target(int64_t Ls, int32_t sink, int32_t lag, double target_C);

/*
 * Bytes of workspace needed: the status block plus, for lagkv_compress_append(), one counter
 * per sequence (rounded up to 256 bytes) and room for max_new_chunks*k kept indices per
 * (b, h).  Pass 0 for prefill / gather only.
 */
size_t lagkv_workspace_bytes(lagkv_plan_t plan, int32_t max_new_chunks);

/* Clear the status block and the append counters (async memset on the stream).  Call once
 * per workspace; the kernels leave the counters at zero. */
int lagkv_workspace_init(lagkv_plan_t plan, void *workspace, size_t workspace_bytes,
                         void *cuda_stream);

/*
 * One-shot compression of a freshly prefilled cache (first bullet of Section 2.2; Eq. 7-12).
 * Every sequence has S_in rows.  Out of place; K, V are not modified and may not alias
 * the outputs.  With L_R = lagkv_compressed_len(plan, S_in, -1):
 *   K_out, V_out [B, H, L_R, D] bf16 contiguous: sink rows, then for p = 0..n-2 the k kept
 *                rows of partition p in ascending position, then the window rows.
 *                Both NULL = indices only.
 *   idx_out      [B, H, L_R] int32 or NULL: source row of every output row.
 *   scores_out   [B, H, (n-1)*L] fp32 or NULL: final score (Eq. 11) of every token of a
 *                compressed partition.
 * S_in < S + 2L is not an error: the pass is the identity (L_R = S_in).
 * Asynchronous on cuda_stream (a cudaStream_t, NULL = default stream).
 */
int lagkv_compress_prefill(lagkv_plan_t plan, const void *K, const void *V, int64_t S_in,
                           void *K_out, void *V_out, int32_t *idx_out, float *scores_out,
                           void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * lagkv_compress_prefill() for caches that live in HOST memory (the same pass, Section 2.2,
 * Eq. 7-12; the paper has no counterpart for the transfer).  K_host, V_host [B, H, S_in, D]
 * and the outputs K_out_host, V_out_host [B, H, L_R, D], idx_out_host [B, H, L_R] are HOST
 * pointers, contiguous, pinned if the copies are to overlap (pageable memory works, slower);
 * the plan's strides must be 0.  The B sequences are cut into chunks of chunk_B (B % chunk_B
 * == 0); each chunk is copied to the device, compressed and copied back, on three internal
 * streams with two staging slots so that copies in both directions overlap the kernel.
 *   staging    caller-owned DEVICE memory, 256-byte aligned, at least
 *              lagkv_host_staging_bytes(plan, S_in, chunk_B) bytes (0 = bad arguments)
 *   workspace  as for lagkv_compress_prefill()
 * Nothing is allocated on the device; streams and events are created once per plan on the
 * first call and freed by lagkv_plan_destroy().  Ordered after the work already on
 * cuda_stream; cuda_stream waits for the last copy, so a synchronise on it (or
 * lagkv_read_status) makes the host buffers valid.  The host does not block.  Calls on one
 * plan are enqueued one at a time (internal lock) and must use the same cuda_stream if they
 * share staging memory.
 */
size_t lagkv_host_staging_bytes(lagkv_plan_t plan, int64_t S_in, int32_t chunk_B);
int lagkv_compress_prefill_host(lagkv_plan_t plan, const void *K_host, const void *V_host, int64_t S_in,
                                void *K_out_host, void *V_out_host, int32_t *idx_out_host,
                                int32_t chunk_B, void *staging, size_t staging_bytes, void *workspace,
                                size_t workspace_bytes, void *cuda_stream);

/*
 * Incremental (recursive) compression during decode or chunked prefill (Section 2.2,
 * bullets 2-4; Fig. 1).  In place on caches [B, H, S_cap, D] (the plan's strides, 0 =
 * contiguous for S_cap).  seq_len[B] and static_len[B] are DEVICE int32 arrays: rows
 * [0, static_len[b]) are the sink plus everything kept so far, rows up to seq_len[b] are
 * valid.  For every sequence whose rest = seq_len - static_len is at least 2L the n-1
 * oldest partitions are scored against their successors, their k kept rows are packed
 * behind the static part, the window (last full partition + remainder) is moved down
 * behind them, and the call sets static_len += (n-1)*k, seq_len = static_len + L + rem.
 * Other sequences are left untouched (decided on the device: no host sync).  The call is
 * always the same single launch with the same arguments, so it may be captured into a CUDA
 * graph once and replayed after every decoded token.
 *   max_new_chunks  capacity: a sequence with n-1 > max_new_chunks is left untouched and
 *                   LAGKV_ECAPACITY is recorded in the status block.
 *   idx_out     [B, H, max_new_chunks*k] int32 or NULL: pre-call positions of the rows
 *               kept by this call (entries of skipped sequences are not written).
 *   scores_out  [B, H, max_new_chunks*L] fp32 or NULL.
 * The workspace must have been sized with the same max_new_chunks.
 * With max_new_chunks == 1 (decode: at most one partition completes per call) and at most
 * sm_count (b, h) units the launch is a grid of thread-block clusters, one cluster per unit,
 * which keeps the window in shared memory between its two uses; it is still one launch.
 */
int lagkv_compress_append(lagkv_plan_t plan, void *K_cache, void *V_cache, int64_t S_cap,
                          int32_t *seq_len, int32_t *static_len, int32_t max_new_chunks,
                          int32_t *idx_out, float *scores_out, void *workspace,
                          size_t workspace_bytes, void *cuda_stream);

/*
 * Paged caches (block tables).  The method itself (Section 2.2) only speaks of a cache of n
 * rows per head; serving engines store that cache as fixed-size pages drawn from a pool, with a
 * table per sequence saying which page holds which rows.  K_pool / V_pool are DEVICE pointers to
 * pools addressed as
 *     pool + block_table[b*max_blocks + s/page_size]*stride_page + h*stride_h + (s%page_size)*stride_s + d
 * (the same table and strides for K and V).  A stride given as 0 means dense
 * [num_pages, H_kv, page_size, D].  With layers folded into B, sequence b's table row simply
 * names pages of its own layer.  The plan's own strides must be 0.
 */
typedef struct {
    const int32_t *block_table; /* DEVICE int32 [B, max_blocks], 4-byte aligned               */
    int32_t max_blocks;         /* entries per sequence; max_blocks*page_size >= rows addressed */
    int32_t page_size;          /* rows per page: a power of two, >= 16                        */
    int64_t stride_page;        /* elements between pages          (0 = H_kv*stride_h)         */
    int64_t stride_h;           /* elements between heads in a page (0 = page_size*stride_s)   */
    int64_t stride_s;           /* elements between rows in a page  (0 = D); all three strides
                                   multiples of 16 bytes                                       */
} lagkv_paged_layout;

/*
 * lagkv_compress_prefill() reading a paged cache (same pass, Section 2.2, Eq. 7-12): every
 * sequence has S_in rows; the outputs are contiguous as there.  Runs on the kernel family that
 * looks rows up page by page (a tile that straddles a page boundary is fetched in two copies).
 */
int lagkv_compress_prefill_paged(lagkv_plan_t plan, const void *K_pool, const void *V_pool,
                                 const lagkv_paged_layout *layout, int64_t S_in, void *K_out, void *V_out,
                                 int32_t *idx_out, float *scores_out, void *workspace, size_t workspace_bytes,
                                 void *cuda_stream);

/*
 * lagkv_compress_append() in place on a paged cache (Section 2.2, bullets 2-4; Fig. 1): kept rows
 * and the window are moved down inside the sequence's own pages, seq_len / static_len are
 * updated as there.  A sequence may hold at most max_blocks*page_size rows.  Pages that lie wholly
 * behind the new seq_len[b] hold no valid rows any more; giving them back to the pool is the
 * caller's business (the table is not modified).
 */
int lagkv_compress_append_paged(lagkv_plan_t plan, void *K_pool, void *V_pool, const lagkv_paged_layout *layout,
                                int32_t *seq_len, int32_t *static_len, int32_t max_new_chunks, int32_t *idx_out,
                                float *scores_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * lagkv_compress_append() for callers that have no device memory to give as a workspace.
 * (The paper has no counterpart: this is a property of the library, not of the method.)
 *
 * Who needs it: code that runs where allocating is off the table -- a decode loop inside a
 * serving engine whose memory pool is already carved up, a plug-in called from someone
 * else's stream callback or capture region, a host that forbids cudaMalloc after start-up
 * because it would synchronise the device.  Such a caller cannot produce the workspace
 * that lagkv_compress_append() wants, so the library brings its own: a fixed array of
 * LAGKV_NOALLOC_SCRATCH_BYTES bytes inside the library image.  Every GPU that loads the
 * library holds one copy of it until the process exits.
 *
 * Arguments are those of lagkv_compress_append() minus workspace / workspace_bytes, plus
 *   status_out  DEVICE int32[4] or NULL: receives the status block of this call (same
 *               meaning as lagkv_read_status(): [0] first device-side status, [1] detail,
 *               [2] zero-range channel count), written on cuda_stream after the kernels.
 *               With NULL the block stays in the built-in array until the next call on that
 *               device clears it: read it before then with lagkv_read_status(plan, NULL, ...),
 *               or a device-side LAGKV_ECAPACITY / LAGKV_EINVAL / LAGKV_ETIMEOUT of this call
 *               goes unnoticed.
 * The call allocates nothing and frees nothing; it enqueues a small memset (status block and
 * counters), the append kernel and, if asked, a 16-byte device-to-device copy.
 *
 * Limit: 256 + 256*ceil(B/64) + B*H_kv*max_new_chunks*k*4 bytes must not exceed
 * LAGKV_NOALLOC_SCRATCH_BYTES when idx_out is NULL (the kept positions are parked in the
 * scratch); with idx_out given only the first two terms (status block, one counter per
 * sequence) are used.  Beyond the limit the call returns
 * LAGKV_ENOALLOC_LIMIT and touches nothing.
 *
 * First call on a device: the library looks up the device address of its array (once per
 * device, with that device current).  Make that first call outside any stream capture.
 *
 * Sharing: all calls on a device use the same array, and the array keeps whatever the last
 * call left in it.  The status block is cleared at the start of every call; the kept
 * positions are rewritten before they are read.  Two calls that overlap on the GPU (two
 * streams, no dependency between them) race on the array: order them.
 */
#define LAGKV_NOALLOC_SCRATCH_BYTES 1048576
int lagkv_compress_append_noalloc(lagkv_plan_t plan, void *K_cache, void *V_cache, int64_t S_cap,
                                  int32_t *seq_len, int32_t *static_len, int32_t max_new_chunks,
                                  int32_t *idx_out, float *scores_out, int32_t *status_out,
                                  void *cuda_stream);

/*
 * Row gather, the separable part of the compaction (Fig. 1):
 *   K_out[b,h,j,:] = K[b,h,idx[b,h,j],:],  same for V,  j < n_idx.
 * K, V use the plan's strides with S_in rows; outputs are contiguous [B, H, n_idx, D].
 * V / V_out may both be NULL.  idx is a DEVICE int32 array [B, H, n_idx]; every entry
 * must lie in [0, S_in) -- entries outside are skipped and LAGKV_EINVAL is recorded in
 * the status block when a workspace is given (workspace may be NULL).
 */
int lagkv_gather(lagkv_plan_t plan, const void *K, const void *V, int64_t S_in,
                 const int32_t *idx, int64_t n_idx, void *K_out, void *V_out, void *workspace,
                 void *cuda_stream);

/* lagkv_gather() reading a paged cache (see lagkv_paged_layout); outputs contiguous as there. */
int lagkv_gather_paged(lagkv_plan_t plan, const void *K_pool, const void *V_pool, const lagkv_paged_layout *layout,
                       int64_t S_in, const int32_t *idx, int64_t n_idx, void *K_out, void *V_out, void *workspace,
                       void *cuda_stream);

/*
 * ---- Attention over the cache ---------------------------------------------------------------
 * The compress pass shortens a cache so that the attention reading it gets cheaper; the entry
 * points from here on are that attention, the choice of blocks it may be limited to, and the pages
 * the pass frees.  They take the same plan (its B, H_kv, D, strides, dtype and device; sink, lag and
 * keep_ratio play no part) and the same caches, one layer per call.
 *
 * Queries: T tokens per sequence, H_q heads; query head h reads KV head h / (H_q / H_kv).  Q and the
 * output are bf16 for bf16 and fp8 caches, fp16 for fp16 caches.  Sums of products of queries and keys,
 * softmax statistics and sums are fp32; probabilities are rounded to the 16-bit type of the matrix
 * products (fp16 for fp8 caches, whose rows widen to fp16 exactly), each by half a step of it.  Over fp8
 * caches a row of queries becomes fp16, too, after a power of two has brought its largest element to
 * [2^8, 2^9): elements below 2^-25 of that one lose bits, at most 2^-33 of it.
 */
typedef struct {
    int32_t T;         /* query tokens per sequence, 1..64                                      */
    int32_t H_q;       /* query heads: H_kv times 1..64                                         */
    double scale;      /* factor of q.k before the softmax, > 0; 0 = 1/sqrt(D)                  */
    double k_scale;    /* what a stored K element of 1 stands for (fp8 caches), > 0; 0 = 1;     */
                       /* scale*k_scale*log2(e) and v_scale are finite in fp32                  */
    double v_scale;    /* the same for V                                                        */
    int64_t stride_b;  /* strides of Q [B, T, H_q, D] in elements, multiples of 8; 0 = dense    */
    int64_t stride_t;  /* over the dimension inside; channel stride 1, 16-byte aligned base     */
    int64_t stride_h;
} lagkv_query;

/*
 * Bytes of workspace for lagkv_attend_tree() (blocks = keep = 0) or lagkv_attend_blocks() (blocks =
 * blocks per sequence of its bounds, keep as in its choice) with up to T tokens and H_q heads; 0 = bad
 * arguments.  A workspace may serve every smaller call, tree and blocks alike, one at a time: calls (or
 * replayed graphs) that may overlap need workspaces of their own.  256-byte aligned; starts with a
 * status block, cleared once with lagkv_attend_workspace_init() (async on the stream), that
 * lagkv_read_status() reads.  LAGKV_ETIMEOUT there: a wait inside a kernel was given up, the results of
 * that call are not valid.
 */
size_t lagkv_attend_workspace_bytes(lagkv_plan_t plan, int32_t T, int32_t H_q, int64_t blocks, int32_t keep);
int lagkv_attend_workspace_init(lagkv_plan_t plan, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Attention of a tree of drafted tokens (T = 1: an ordinary decode step).  seq_len[B] (DEVICE int32)
 * counts the valid rows of each sequence, the drafted tokens' own rows included: those are its last
 * draft_len[b] rows (DEVICE int32 [B], 0..T; NULL = T everywhere).  Token t of sequence b sees row r when
 *     r < seq_len[b] - draft_len[b]          (everything before the draft), or
 *     r = seq_len[b] - draft_len[b] + j and bit j of tree_mask[b*T + t] is set.
 * tree_mask (DEVICE uint64 [B, T]): NULL = a chain, token t sees drafted rows 0..t.  Rows at or behind
 * seq_len[b], and drafted rows a token does not see, never reach it, whatever they hold.
 *   out      [B, T, H_q, D] contiguous; lse_out fp32 [B, T, H_q] or NULL: natural log of the sum of
 *            exp(scale*k_scale*q.k) over the rows seen.  A token that sees no row, and the padding
 *            tokens t >= draft_len[b], get out = 0 and lse = -infinity.
 * seq_len[b] = 0 is an empty slot of the batch (no tokens when draft_len is NULL).
 * seq_len[b] outside [0, S_cap], draft_len[b] outside [0, T] or above seq_len[b]: that sequence counts as
 * without tokens and LAGKV_EINVAL is recorded in the status block.
 * Two launches, the same with the same arguments for every length, so the call may be captured into a CUDA
 * graph.  The same call gives the same bits.
 */
int lagkv_attend_tree(lagkv_plan_t plan, const lagkv_query *query, const void *Q, const void *K, const void *V,
                      int64_t S_cap, const int32_t *seq_len, const int32_t *draft_len, const uint64_t *tree_mask,
                      void *out, float *lse_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * The same on a paged cache.  num_pages = pages of the pools: a table entry outside [0, num_pages) that
 * a sequence's length reaches is not read; its rows count as not there and LAGKV_EINVAL is recorded.
 */
int lagkv_attend_tree_paged(lagkv_plan_t plan, const lagkv_query *query, const void *Q, const void *K_pool,
                            const void *V_pool, const lagkv_paged_layout *layout, int64_t num_pages,
                            const int32_t *seq_len, const int32_t *draft_len, const uint64_t *tree_mask, void *out,
                            float *lse_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Keep the accepted path of each tree: with base = seq_len[b] - draft_len[b] the rows
 * base + accepted[b*T + j], j < n_accepted[b], move to base + j in K and V (every KV head), and
 * seq_len[b] becomes base + n_accepted[b].  accepted (DEVICE int32 [B, T]) ascends strictly inside
 * [0, draft_len[b]).  A sequence whose lengths or path are not of that form is left untouched and
 * LAGKV_EINVAL is recorded.  draft_len as above (NULL: an empty slot, seq_len[b] = 0, has no draft and takes
 * n_accepted[b] = 0), T 1..64.  The workspace needs its status block only.
 */
int lagkv_tree_commit(lagkv_plan_t plan, void *K_cache, void *V_cache, int64_t S_cap, int32_t *seq_len,
                      const int32_t *draft_len, int32_t T, const int32_t *accepted, const int32_t *n_accepted,
                      void *workspace, size_t workspace_bytes, void *cuda_stream);
int lagkv_tree_commit_paged(lagkv_plan_t plan, void *K_pool, void *V_pool, const lagkv_paged_layout *layout,
                            int64_t num_pages, int32_t *seq_len, const int32_t *draft_len, int32_t T,
                            const int32_t *accepted, const int32_t *n_accepted, void *workspace,
                            size_t workspace_bytes, void *cuda_stream);

/*
 * Bounds of the blocks of a cache: block j of a (sequence, KV head) is its rows [j*block_rows,
 * (j+1)*block_rows) below seq_len[b]; bounds[b][h][j][0] and [1] are the per-channel minimum and maximum of
 * their K rows, in the plan's storage format (exact), [B, H_kv, blocks, 2, D] contiguous.
 *   from_len  DEVICE int32 [B] or NULL (0): rows below it have not changed since the bounds were last
 *             written; blocks that end at or before it are left as they are.  After a token has been
 *             appended this is the old length, after lagkv_compress_append() the static_len before it.
 *   block_rows  16, 32, 64 or 128; blocks*block_rows >= S_cap.
 * Blocks behind the last row are not written.  NaN in a seen K row leaves that channel undefined.
 */
int lagkv_block_bounds(lagkv_plan_t plan, const void *K, int64_t S_cap, const int32_t *from_len,
                       const int32_t *seq_len, int32_t block_rows, void *bounds, int64_t blocks, void *workspace,
                       size_t workspace_bytes, void *cuda_stream);
int lagkv_block_bounds_paged(lagkv_plan_t plan, const void *K_pool, const lagkv_paged_layout *layout,
                             int64_t num_pages, const int32_t *from_len, const int32_t *seq_len, int32_t block_rows,
                             void *bounds, int64_t blocks, void *workspace, size_t workspace_bytes, void *cuda_stream);

typedef struct {
    int32_t block_rows;     /* rows per block of the bounds: 16, 32, 64 or 128                          */
    int32_t keep;           /* blocks each (token, KV head) attends to, at most 4096                    */
    int32_t sink_blocks;    /* of these, the first ones of the sequence, always kept ...                */
    int32_t recent_blocks;  /* ... and the last ones; sink_blocks + recent_blocks <= keep               */
    int64_t blocks;         /* blocks per (sequence, KV head) of the bounds, at most 24576              */
} lagkv_block_choice;

/*
 * Attention to a choice of blocks.  Token t of sequence b sees the rows below end = seq_len[b] - (T-1-t)
 * (its own row is the last of them) that lie in the blocks chosen for it and for each KV head: the
 * first sink_blocks and the last recent_blocks of its ceil(end/block_rows) blocks, and of the others
 * those with the largest score
 *     max over the query heads g of the KV head of  sum_c max(q_gc*min_c, q_gc*max_c)
 * (no logit of the block is larger), `keep` in all, the lower block among equals.  Scores are summed in
 * 64 bits.  bounds must cover every row below seq_len[b].  Rows at or behind `end` never reach a token.
 *   idx_out  int32 [B, T, H_kv, keep] or NULL: the chosen blocks, ascending, -1 behind the last.
 * seq_len[b] outside [0, S_cap], or in 1..T-1: LAGKV_EINVAL is recorded; such a sequence and an empty one
 * (seq_len[b] = 0) get out = 0, lse = -infinity, idx = -1.
 * out, lse_out and the rest as for lagkv_attend_tree().  Four launches.
 */
int lagkv_attend_blocks(lagkv_plan_t plan, const lagkv_query *query, const lagkv_block_choice *choice, const void *Q,
                        const void *K, const void *V, int64_t S_cap, const int32_t *seq_len, const void *bounds,
                        void *out, float *lse_out, int32_t *idx_out, void *workspace, size_t workspace_bytes,
                        void *cuda_stream);
int lagkv_attend_blocks_paged(lagkv_plan_t plan, const lagkv_query *query, const lagkv_block_choice *choice,
                              const void *Q, const void *K_pool, const void *V_pool, const lagkv_paged_layout *layout,
                              int64_t num_pages, const int32_t *seq_len, const void *bounds, void *out, float *lse_out,
                              int32_t *idx_out, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * ---- Caches in 8 bits with block scales --------------------------------------------------------
 * A cache for a plan of 16-bit format that stores 8-bit codes and one fp32 scale per (sequence, KV head, block of
 * block_rows rows), for K and for V: row r stands for scale[b][h][r/block_rows] * codes.  Rows are quantised as they
 * are written, read back in 16 bits where the compress pass is to run on them again, and attended to
 * as they are.  plan: B, H_kv, D, dtype (bf16 or fp16: the 16-bit side, queries and outputs) and device as everywhere;
 * its strides are those of the 16-bit cache that lagkv_quant_read() fills (and have to be 0 for paged caches).
 */
enum lagkv_quant_format {
    LAGKV_QUANT_INT8 = 0, /* signed whole numbers, -127..127 as written here                     */
    LAGKV_QUANT_E4M3 = 1  /* e4m3 as in LAGKV_DTYPE_FP8_E4M3; scales written here are powers of two */
};

typedef struct {
    void *K, *V;          /* DEVICE codes, 16-byte aligned: [B, H_kv, S_cap, D], or pools of pages    */
    float *K_scale;       /* DEVICE fp32 [B, H_kv, blocks], of K and of V; >= 0, finite               */
    float *V_scale;
    int32_t format;       /* enum lagkv_quant_format                                                  */
    int32_t block_rows;   /* 16, 32, 64 or 128; on paged caches at most page_size                     */
    int64_t blocks;       /* blocks*block_rows >= rows a sequence may have                            */
    int64_t stride_b;     /* strides of the codes in bytes, multiples of 16; 0 = dense, as for other  */
    int64_t stride_h;     /* caches; 0 on paged caches, whose layout carries them (in bytes)          */
    int64_t stride_s;
} lagkv_quant_cache;

/* Rows to write: K, V [B, H_kv, T, D] in the plan's 16-bit format, any strides with channel stride 1. */
typedef struct {
    int32_t T;            /* rows per (sequence, KV head) of K and V                                  */
    int32_t at_positions; /* 0: position p of the cache is row p - from_len[b]; else row p (T > every
                             position written), as when a 16-bit cache is quantised                   */
    const int32_t *take;  /* NULL, or DEVICE int32 [B, take_heads, take_rows]: position from_len[b] + i
                             is row take[..][i] (then at_positions plays no part): the idx_out of
                             lagkv_compress_prefill() writes the kept rows straight from the raw cache,
                             a list of accepted tokens those of a draft                               */
    int32_t take_heads;   /* 1 (the same for every KV head) or H_kv                                   */
    int32_t take_rows;
    int64_t stride_b;     /* in elements, multiples of 8; 0 = dense                                   */
    int64_t stride_h;
    int64_t stride_t;
} lagkv_quant_source;

/*
 * Write rows [from_len[b], seq_len[b]) of each sequence (DEVICE int32 [B]; from_len NULL = 0; the caller's lengths are not
 * changed).  With a = the largest magnitude of the rows of a block that the call writes,
 *     int8:  f = max(a/127, 2^-126), a/127 correctly rounded to fp32; code = x/s, nearest whole number, ties to even
 *     e4m3:  f = max(the least power of two with a <= 448*f, 2^-126); code = the nearest e4m3 to x/s
 * (f = 0 where a = 0).  A block that begins at or behind from_len[b] gets s = f.  One that holds older rows gets
 * s = max(f, its scale); where that is larger the older codes become code*(old scale)/s, rounded again.  The codes are those of
 * exact quotients.  Other blocks, and rows behind seq_len[b], stay as they are.
 * Values that are not finite: LAGKV_EINVAL is recorded; they do not count in a, infinities become the largest code, NaN 0.
 * Under a scale of 0 every code is 0, that of an infinity too (a block whose new rows hold no finite value but zeros).
 * Refused (LAGKV_EINVAL recorded, the sequence untouched): lengths outside 0 <= from_len <= seq_len <= S_cap, more new
 * rows than T (take_rows), positions behind T with at_positions.  A take entry outside [0, T): recorded, that row is 0.
 * A page outside the pool: recorded, its block is left out.  No page may be written through two table entries.
 * One launch; the workspace needs its status block only, and any workspace of the plan will do.
 */
int lagkv_quant_write(lagkv_plan_t plan, const lagkv_quant_cache *cache, int64_t S_cap, const lagkv_quant_source *source,
                      const void *K, const void *V, const int32_t *from_len, const int32_t *seq_len, void *workspace,
                      size_t workspace_bytes, void *cuda_stream);
int lagkv_quant_write_paged(lagkv_plan_t plan, const lagkv_quant_cache *cache, const lagkv_paged_layout *layout,
                            int64_t num_pages, const lagkv_quant_source *source, const void *K, const void *V,
                            const int32_t *from_len, const int32_t *seq_len, void *workspace, size_t workspace_bytes,
                            void *cuda_stream);

/*
 * Read rows back in the plan's 16-bit format: scale*code in fp32, rounded once more to 16 bits (values beyond its largest
 * become that).
 *   idx NULL: K_out, V_out are caches [B, H_kv, rows_out, D] with the plan's strides (0 = dense); rows [from_len[b], seq_len[b])
 *             go to the same positions there, others stay as they are.  rows_out >= every seq_len[b].
 *   idx       DEVICE int32 [B, H_kv, rows_out], from_len NULL: row i of the dense outputs [B, H_kv, rows_out, D] is row
 *             idx[b][h][i], in [0, seq_len[b]); other entries are recorded and leave their row as it is.
 * K_out or V_out may be NULL.  Lengths that do not fit: LAGKV_EINVAL recorded, nothing read.  A page outside the pool:
 * recorded, its rows stay as they are.  One launch; the workspace needs its status block only.
 */
int lagkv_quant_read(lagkv_plan_t plan, const lagkv_quant_cache *cache, int64_t S_cap, const int32_t *from_len,
                     const int32_t *seq_len, const int32_t *idx, int64_t rows_out, void *K_out, void *V_out,
                     void *workspace, size_t workspace_bytes, void *cuda_stream);
int lagkv_quant_read_paged(lagkv_plan_t plan, const lagkv_quant_cache *cache, const lagkv_paged_layout *layout,
                           int64_t num_pages, const int32_t *from_len, const int32_t *seq_len, const int32_t *idx,
                           int64_t rows_out, void *K_out, void *V_out, void *workspace, size_t workspace_bytes,
                           void *cuda_stream);

/*
 * lagkv_attend_tree() over such a cache: the same lengths, masks, queries (T, heads, strides, scale; k_scale and v_scale
 * count on top of the block scales), results and errors.  cap > 0 (2^-100 at least): every logit x becomes cap*tanh(x/cap); 0: none.
 * Products are in fp16 (codes are exact in it) with fp32 sums; bf16 queries enter as fp16 after a power of two per row,
 * as over fp8 caches.  K scales multiply the fp32 logits; V scales multiply the probabilities before these are rounded to
 * fp16, relative to a power of two near the largest V scale seen: a row whose probability (of the largest one) times its scale
 * is below 2^-22 of that scale loses bits, 2^-32 of the scale times its code at most.
 * One launch for few short caches, else two; which kernels serve a call goes by its sizes and capacity, not by the lengths.
 * Workspace: lagkv_attend_quant_workspace_bytes() (0 = bad arguments), cleared once with
 * lagkv_attend_workspace_init(); it serves every smaller call, one at a time.
 */
size_t lagkv_attend_quant_workspace_bytes(lagkv_plan_t plan, int32_t T, int32_t H_q);
int lagkv_attend_quant(lagkv_plan_t plan, const lagkv_query *query, double cap, const lagkv_quant_cache *cache, const void *Q,
                       int64_t S_cap, const int32_t *seq_len, const int32_t *draft_len, const uint64_t *tree_mask,
                       void *out, float *lse_out, void *workspace, size_t workspace_bytes, void *cuda_stream);
int lagkv_attend_quant_paged(lagkv_plan_t plan, const lagkv_query *query, double cap, const lagkv_quant_cache *cache,
                             const void *Q, const lagkv_paged_layout *layout, int64_t num_pages, const int32_t *seq_len,
                             const int32_t *draft_len, const uint64_t *tree_mask, void *out, float *lse_out,
                             void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * ---- Pages --------------------------------------------------------------------------------
 * A pool of num_pages pages, block tables over it (lagkv_paged_layout; entries are -1 where a sequence
 * has no page) and refs (DEVICE int32 [num_pages]): refs[p] = table entries that name page p, 0 = free.
 * The four calls below keep the three in step; the block table they are given is written.  Pages are
 * handed out lowest first, so the result depends on the state alone.  Tables of several layers (folded
 * into B) may share one pool and one refs.  num_pages < 2^30.
 * Workspace: at least lagkv_pages_workspace_bytes() (0 = bad arguments), 256-byte aligned, cleared once
 * with lagkv_pages_workspace_init(), for one call at a time; lagkv_read_status() reads its status block.
 */
size_t lagkv_pages_workspace_bytes(lagkv_plan_t plan, int64_t num_pages);
int lagkv_pages_workspace_init(lagkv_plan_t plan, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Give back the pages that lie wholly at or behind row keep_len[b] (DEVICE int32 [B]; 0 frees the
 * sequence): their entries become -1 and refs go down by one each.  After lagkv_compress_append_paged()
 * keep_len = seq_len frees what the pass has emptied.  keep_len[b] outside [0, max_blocks*page_size], an
 * entry outside the pool, or a page that refs counts as free: recorded as LAGKV_EINVAL and left alone.
 */
int lagkv_pages_release(lagkv_plan_t plan, int32_t *block_table, int32_t max_blocks, int32_t page_size,
                        int64_t num_pages, int32_t *refs, const int32_t *keep_len, void *workspace,
                        size_t workspace_bytes, void *cuda_stream);

/*
 * Room for want_len[b] rows (DEVICE int32 [B]): every entry of the first ceil(want_len[b]/page_size) blocks
 * that is negative gets a free page, in the order (sequence, block); pages already there stay, and
 * so do those behind.  Too few free pages: LAGKV_ECAPACITY is recorded and nothing changes.  want_len[b]
 * outside [0, max_blocks*page_size]: LAGKV_EINVAL is recorded, that sequence gets nothing.
 */
int lagkv_pages_reserve(lagkv_plan_t plan, int32_t *block_table, int32_t max_blocks, int32_t page_size,
                        int64_t num_pages, int32_t *refs, const int32_t *want_len, void *workspace,
                        size_t workspace_bytes, void *cuda_stream);

/*
 * Fork sequences: for i < n (at most B) sequence dst[i], which holds no pages, becomes a copy of sequence
 * src[i] (DEVICE int32 [n] each), seq_len and static_len (DEVICE int32 [B]) included.  Pages wholly below
 * min(seq_len, static_len) are shared: those rows are never rewritten, not by the compress pass, not by
 * new rows, not by lagkv_tree_commit().  The others are copied to free pages, whole, in the order (i, block), so
 * that both sequences may go on on their own.  (A cache that is never compressed:
 * static_len = seq_len, drafted rows not counted.)
 * A pair is refused (LAGKV_EINVAL recorded, the others done) when an index is outside [0, B), dst[i] holds a
 * page or is the target of an earlier pair, or a page that src[i]'s length needs is not a counted page
 * of the pool.  Too few free pages: LAGKV_ECAPACITY is recorded and nothing changes.  Two launches.
 */
int lagkv_pages_fork(lagkv_plan_t plan, void *K_pool, void *V_pool, const lagkv_paged_layout *layout,
                     int64_t num_pages, int32_t *refs, int32_t *seq_len, int32_t *static_len, const int32_t *src,
                     const int32_t *dst, int32_t n, void *workspace, size_t workspace_bytes, void *cuda_stream);

/*
 * Make the pool dense: with `live` pages in use, each one numbered live or higher moves, in ascending
 * order, to the lowest free numbers; K, V, refs and the block table follow.  Afterwards the pages [live,
 * num_pages) are free.  live_out: DEVICE int32 [1].  Every table that names pages of this pool has to be
 * in the call.  An entry that names a page which refs does not count, or none of the pool: recorded as
 * LAGKV_EINVAL, and it becomes -1, since its number may be another sequence's page afterwards.
 */
int lagkv_pages_compact(lagkv_plan_t plan, void *K_pool, void *V_pool, const lagkv_paged_layout *layout,
                        int64_t num_pages, int32_t *refs, int32_t *live_out, void *workspace, size_t workspace_bytes,
                        void *cuda_stream);

/*
 * Synchronise cuda_stream, copy the status block to the host and clear it.  workspace == NULL
 * names the status block of the library's built-in scratch on the plan's device (the one
 * lagkv_compress_append_noalloc() uses).
 * host_status[0] = first device-side lagkv_status recorded since the last read (0 = none),
 * host_status[1] = detail (block index), host_status[2] = count of zero-range reference
 * channels seen, host_status[3] = reserved.  Returns host_status[0], or LAGKV_ECUDA.
 */
int lagkv_read_status(lagkv_plan_t plan, void *workspace, void *cuda_stream,
                      int32_t host_status[4]);

/*
 * Launch shape the plan uses for a prefill of S_in rows: info[0] = grid, info[1] = block
 * threads, info[2] = dynamic shared memory bytes, info[3] = kernel launches per call,
 * info[4] = kernel family (0 = identity copy, 1 = uniform kernel, 2 = warp-specialised
 * kernel, 3 = pair kernel), info[5] = kernel family lagkv_compress_prefill_paged() uses for
 * the same call (1 or 2; 0 for the identity copy).
 */
int lagkv_launch_info(lagkv_plan_t plan, int64_t S_in, int32_t info[6]);

/*
 * Tuning override of the launch shape: warps per CTA (2, 4 or 8 = the uniform kernel, used
 * for prefill and append alike; 12 = the warp-specialised prefill kernel with 8 streaming,
 * 3 select and 1 copy warp; LAGKV_TUNE_PAIRS = the prefill kernel for partitions of at most
 * 512 rows, four K/V warp pairs with an epilogue warp each, LagKV only; the last two leave
 * the append shape alone), rows per staged tile
 * (16 or 32), ring stages per streaming warp (2..8) and resident CTAs per SM to size the
 * prefill grid for (>= 1; must be 1 with 12 warps).  A value of 0 keeps the current
 * choice.  Returns LAGKV_EUNSUPPORTED for a combination that was not compiled or does not
 * fit shared memory.
 */
#define LAGKV_TUNE_PAIRS 100
/*
 * warps = LAGKV_TUNE_APPEND_CLUSTER (4 warps per CTA) or LAGKV_TUNE_APPEND_CLUSTER8 (8 warps,
 * head_dim 128 only) shapes the kernel of one-partition appends (lagkv_compress_append with
 * max_new_chunks == 1, LagKV scoring) instead: tile_rows = row splits per tensor (1, 2 or 4: a
 * cluster of 2, 4 or 8 CTAs per (b, h) unit), stages = ring stages (2..4), ctas_per_sm = CTAs
 * per SM to leave room for (1..4; fewer resident rows of the window when they do not all fit,
 * which only a split of 1 allows).  The prefill shape is left alone.
 */
#define LAGKV_TUNE_APPEND_CLUSTER 101
#define LAGKV_TUNE_APPEND_CLUSTER8 102
int lagkv_plan_tune(lagkv_plan_t plan, int32_t warps, int32_t tile_rows, int32_t stages,
                    int32_t ctas_per_sm);

/*
 * Self-test of the failure path: launches one warp that waits, with the same bounded wait the
 * compress kernels use, on a barrier nothing will ever complete.  After about limit_ms
 * (1..2000) the wait gives up and LAGKV_ETIMEOUT is recorded in the status block of
 * `workspace` (read it with lagkv_read_status()); the device stays usable.  Asynchronous.
 */
int lagkv_selftest_bounded_wait(lagkv_plan_t plan, void *workspace, int32_t limit_ms, void *cuda_stream);

const char *lagkv_status_string(int status);
const char *lagkv_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LAGKV_H_ */
