// Attention over a (compressed) KV cache -- sm_100a device code.
//
// One query token, or a tree of up to 64 drafted tokens, per sequence (lagkv_attend_tree), or the
// rows of selected blocks only (lagkv_attend_blocks).  For query row m = (token t, query head g of a
// KV head) over the rows r it sees:
//     x_r = scale * q.k_r * log2(e),  p_r = 2^(x_r - ref),  out = sum p_r v_r / sum p_r,
//     lse = ln 2 * (ref + log2 sum p_r),
// one pass over the rows with the running maximum, the running sum and the accumulators in fp32
// registers.  What must be read is every visible row of K and V once per KV head, so the query heads
// of a KV head and the tokens of a tree share the tiles: they are the M rows of the matrix products.
//
// Work is cut on the device, from seq_len: (sequence, KV head, group of M rows) units of 64-row
// tiles, dealt to the CTAs in equal contiguous shares, so ragged batches and a single long sequence
// fill the GPU alike and the same launches with the same arguments serve every length (CUDA graphs).  A unit
// that several CTAs share goes through fp32 partials in the workspace; a kernel launched behind adds
// them in the order of the rows.
#pragma once
#include "lagkv_kernels.cuh"

namespace lagkv {

struct AttendParams {
    const uint8_t* K;
    const uint8_t* V;
    const uint16_t* Q;
    uint16_t* out;         // [B, T, H * G, D]
    float* lse;            // [B, T, H * G] or nullptr
    const int32_t* seq_len;
    const int32_t* draft_len;         // nullptr: T for every sequence
    const unsigned long long* mask;   // [B, T] visible drafted rows; nullptr: a chain (token t sees rows <= t)
    int32_t* status;
    float* partials;       // [grid * 2][MR * (D + 2)]
    int2* shared;          // first and last CTA of each unit
    long long sb, sh, ss, page_stride;  // bytes
    const int32_t* block_table;
    long long num_pages;
    long long q_sb, q_st, q_sh;         // elements
    int B, H, G, T, S_cap, max_blocks, page_shift;
    int mtiles;            // groups of M rows per (sequence, KV head)
    int ctas;              // CTAs of the attention kernel
    int least;             // wide kernel: tiles that a CTA takes at least
    float per_units;       // the other: 1 / (16 units)
    int lead;              // what beginning a unit costs, in tiles: counted when the work is shared out
    float scale_log2, v_scale;
    const int32_t* idx;    // blocks: [B, T, H, keep] ascending block numbers, -1 behind the last
    int keep, block_shift;
};

constexpr int kAttendTile = 64;     // rows of the unit of scheduling (lagkv_attend_kernel)
constexpr int kAttendLead = 6;      // P.lead: 16 caches of 16384 rows in 79 us, 85 with equal shares of the rows
constexpr int kAttendWarps = 4;
constexpr int kWarpRows = 16;       // rows of a warp's tile: never across a page or a block (both >= 16)

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool full) {
    const int n = full ? 16 : 0;  // 0 bytes read: the 16 bytes are zero-filled
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(a)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(a)
                 : "memory");
}
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Arithmetic of the matrix products by storage format.  fp8 rows are widened exactly to fp16; the
// bf16 queries they come with are rounded to fp16 after an exact power-of-two scaling per row.
template <int DT>
struct Mma {  // bf16
    static constexpr float kRefShift = 0.f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
struct MmaHalf {  // fp16: probabilities up to 2^8, so that small ones stay clear of the subnormals
    static constexpr float kRefShift = 8.f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <>
struct Mma<1> : MmaHalf {};
template <>
struct Mma<2> : MmaHalf {};

__device__ __forceinline__ float q_to_float(uint16_t w, bool half) {
    return half ? Elem<1>::lo(w) : Elem<0>::lo(w);
}
// 16-bit output of a batch: fp16 for fp16 caches, bf16 for bf16 and fp8 caches
template <int DT>
__device__ __forceinline__ uint32_t pack_out(float lo, float hi) {
    return DT == 1 ? MmaHalf::pack(lo, hi) : Mma<0>::pack(lo, hi);
}

// ---------------------------------------------------------------------------------- geometry
template <int D_, int DT_, int MT_>
struct AttendGeo {
    static constexpr int D = D_, DT = DT_, MT = MT_;
    static constexpr int EB = Elem<DT_>::EB;
    static constexpr int NW = kAttendWarps, NT = NW * 32;
    static constexpr int MR = 16 * MT;                 // query rows of a unit
    static constexpr int ROWB = D * EB, CPR = ROWB / 16;
    static constexpr int PITCH = ROWB + 16;            // an odd number of 16-byte chunks: ldmatrix without conflicts
    static constexpr int TENSOR = kWarpRows * PITCH;   // one warp's tile of K or of V
    static constexpr int STAGE = 2 * TENSOR;
    static constexpr int STAGES = STAGE * NW * 4 <= 112 * 1024 ? 4 : 3;
    static constexpr int QPITCH = D * 2 + 16;
    static constexpr int RING = NW * STAGES * STAGE;
    static constexpr int EPI = NW * MR * (D + 4) * 4;  // the warps' accumulators, over the ring
    static constexpr int OFF_Q = RING > EPI ? RING : EPI;
    static constexpr int OFF_MASK = OFF_Q + MR * QPITCH;
    static constexpr int OFF_ML = OFF_MASK + MR * 8;               // [NW][MR][2] reference and sum
    static constexpr int OFF_SCALE = OFF_ML + NW * MR * 8;         // [MR]
    static constexpr int OFF_SCAN = OFF_SCALE + MR * 4;            // scheduling scratch
    static constexpr int SMEM = OFF_SCAN + 64 + 8 * NW;
    static constexpr int CTAS_SMEM = (228 * 1024) / (SMEM + 1024);
    static constexpr int CTAS_REGS = (D * MT >= 256) ? 2 : 3;
    static constexpr int CTAS = CTAS_SMEM < CTAS_REGS ? CTAS_SMEM : CTAS_REGS;
    static_assert(CPR * kWarpRows % 32 == 0 && (PITCH / 16) % 2 == 1, "bad geometry");
    static_assert(CTAS >= 1 && SMEM <= 227 * 1024, "does not fit");
};

// One sequence as the scheduler sees it.
struct AttendSeq {
    int len;     // rows below seq_len (0 where the lengths do not describe the cache)
    int tokens;  // drafted tokens (rows len - tokens .. len - 1)
    int tiles;   // TILE-row tiles of each of its units
};
template <int TILE = kAttendTile>
__device__ __forceinline__ AttendSeq attend_seq(const AttendParams& P, int b, bool report) {
    AttendSeq s;
    s.len = __ldg(P.seq_len + b);
    s.tokens = P.draft_len ? __ldg(P.draft_len + b) : s.len == 0 ? 0 : P.T;  // an empty slot of the batch is no error
    if (s.len < 0 || s.len > P.S_cap || s.tokens < 0 || s.tokens > P.T || s.tokens > s.len) {
        if (report) record_status(P.status, ST_EINVAL, b);
        s.len = s.tokens = 0;
    }
    int rows = s.len;
    if (P.idx != nullptr) {
        const int nblk = (s.len + (1 << P.block_shift) - 1) >> P.block_shift;
        rows = min(nblk, P.keep) << P.block_shift;
    }
    if (s.tokens == 0) rows = 0;
    s.tiles = max(1, (rows + TILE - 1) / TILE);  // a unit without rows still writes its zeros
    return s;
}

// a / b for 0 <= a, 0 < b: in 32 bits where they fit, which is what every real batch does
__device__ __forceinline__ long long div_small(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? (long long)(uint32_t(a) / uint32_t(b)) : a / b;
}

// A CTA's share of the tiles: [pos, end) in the order (sequence, unit, tile), where each unit begins with
// P.lead tiles of no rows, so that a CTA which drains one unit and begins another gets fewer rows; `b` and
// `first` are the sequence that holds pos and its first tile.
struct AttendShare {
    long long pos, end, first, per_cta;
    int b;
};
// The part of a share that lies in one unit.
struct AttendPart {
    int u;               // unit of the sequence
    int tile0, n;        // tiles with rows (n = 0: none)
    int step;            // tiles to go on by, those of no rows too
    long long c0, c1;    // first and last CTA that have rows of the unit
};
__device__ __forceinline__ AttendPart attend_part(const AttendParams& P, const AttendShare& sh, int tiles) {
    AttendPart a;
    const int all = tiles + P.lead;
    a.u = int(div_small(sh.pos - sh.first, all));
    const long long begin = sh.first + (long long)a.u * all;
    const int v0 = int(sh.pos - begin);
    a.step = int(min((long long)(all - v0), sh.end - sh.pos));
    a.tile0 = max(0, v0 - P.lead);
    a.n = max(0, v0 + a.step - P.lead - a.tile0);
    a.c0 = div_small(begin + P.lead, sh.per_cta);
    a.c1 = div_small(begin + all - 1, sh.per_cta);
    return a;
}
__device__ __forceinline__ void attend_advance(const AttendParams& P, AttendShare& sh, int step, int tiles, int units_per_seq) {
    sh.pos += step;
    if (sh.pos == sh.first + (long long)units_per_seq * (tiles + P.lead)) {
        sh.first = sh.pos;
        ++sh.b;
    }
}
// `scan`: [NT / 32 + 2] words of shared memory.  Batches of up to NT sequences take one look at the lengths.
template <int NT, int TILE = kAttendTile>
__device__ __forceinline__ AttendShare attend_share(const AttendParams& P, int units_per_seq, long long* scan) {
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    constexpr int NW = NT / 32;
    auto tiles_of = [&](int b, bool report) {
        return b < P.B ? (long long)(attend_seq<TILE>(P, b, report).tiles + P.lead) * units_per_seq : 0ll;
    };
    // inclusive sum over the CTA up to this thread; `all`: over the CTA
    auto sum_up = [&](long long n, long long* all) {
        long long inc = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(~0u, inc, o);
            if (lane >= o) inc += v;
        }
        if (lane == 31) scan[w] = inc;
        __syncthreads();
        *all = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            if (i == w) inc += *all;  // the warps before
            *all += scan[i];
        }
        return inc;
    };
    long long n = tiles_of(tid, blockIdx.x == 0), all, total;
    long long inc = sum_up(n, &all);
    total = all;
    for (int b0 = NT; b0 < P.B; b0 += NT) {
        __syncthreads();
        sum_up(tiles_of(b0 + tid, blockIdx.x == 0), &all);
        total += all;
    }
    AttendShare s;
    // Equal shares, but not so small that joining them takes over: a share of p tiles takes time in p, the joining of a
    // unit's W / p partials in W / p, so p is at least some sqrt(W): with W / 16 the least times measured are met within
    // 10 % (128 channels, one token, one KV head of 20000 rows: 15 us, of 100000: 30; 8 KV heads of 1216: 9.7, 10.4 with
    // W / 6; equal shares took 32, 54 and 12 when joining was slower).  The wide kernel has no registers to spare for
    // this, not even here (102 -> 109 us where it changes no share): P.least.
    s.per_cta = div_small(total + gridDim.x - 1, gridDim.x);
    if constexpr (TILE == kAttendTile) {
        float p;  // approximate: it decides nothing but the shares, and the same way in every CTA
        asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(p) : "f"(float(total) * P.per_units));
        s.per_cta = max((long long)int(p + 0.999f), s.per_cta);
    } else {
        s.per_cta = max((long long)P.least, s.per_cta);
    }
    s.pos = s.per_cta * blockIdx.x;
    s.end = s.pos + s.per_cta < total ? s.pos + s.per_cta : total;
    s.b = 0;
    s.first = 0;
    if (s.pos >= total) {
        s.pos = s.end = total;
        return s;  // uniform over the CTA
    }
    long long* found = scan + NW;
    long long base = 0;
    for (int b0 = 0;;) {
        if (n > 0 && s.pos >= base + inc - n && s.pos < base + inc) {
            found[0] = b0 + tid;
            found[1] = base + inc - n;
        }
        __syncthreads();
        if (P.B <= NT) break;
        // more sequences than threads: the groups one after the other until one holds pos
        if (b0 == 0) {  // `all` is the last group's: the first one's again
            inc = sum_up(n, &all);
            __syncthreads();
        }
        base += all;
        if (base > s.pos) break;
        b0 += NT;
        n = tiles_of(b0 + tid, false);
        inc = sum_up(n, &all);
    }
    s.b = int(found[0]);
    s.first = found[1];
    return s;
}

// Byte offset of the 16 rows from `row0` on of one unit (row0 is a multiple of 16); -1: a page number
// outside the pool (recorded; the rows count as not there).
__device__ __forceinline__ long long attend_offset(const AttendParams& P, int b, int h, int row0) {
    if (P.block_table == nullptr) return (long long)b * P.sb + (long long)h * P.sh + (long long)row0 * P.ss;
    const int page = __ldg(P.block_table + (long long)b * P.max_blocks + (row0 >> P.page_shift));
    if (page < 0 || page >= P.num_pages) {
        record_status(P.status, ST_EINVAL, b);
        return -1;
    }
    return (long long)page * P.page_stride + (long long)h * P.sh + (long long)(row0 & ((1 << P.page_shift) - 1)) * P.ss;
}

// The finished result of N (4 or 8) channels d .. of query row m of a unit.
template <int D, int DT, int N>
__device__ __forceinline__ void attend_write(const AttendParams& P, int b, int h, int t0, int m0, int tokens, int m, int d,
                                             const float (&o)[N], float ref, float sum) {
    const int row = m0 + m, t = t0 + row / P.G, g = row % P.G;
    const long long at = (((long long)b * P.T + t) * P.H + h) * P.G + g;
    const bool live = t < tokens && sum != 0.f;  // NaN sums stay: they compare unequal to 0
    const float inv = live ? P.v_scale / sum : 0.f;
    uint32_t v[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = live ? pack_out<DT>(o[2 * i] * inv, o[2 * i + 1] * inv) : 0u;
    if constexpr (N == 8)
        *reinterpret_cast<uint4*>(P.out + at * D + d) = make_uint4(v[0], v[1], v[2], v[3]);
    else
        *reinterpret_cast<uint2*>(P.out + at * D + d) = make_uint2(v[0], v[1]);
    if (d == 0 && P.lse) P.lse[at] = live ? 0.69314718055994531f * (ref + log2f(sum)) : -INFINITY;
}

template <int D, int DT, int MT>
__global__ void __launch_bounds__(kAttendWarps * 32, AttendGeo<D, DT, MT>::CTAS)
lagkv_attend_kernel(const __grid_constant__ AttendParams P) {
    using G = AttendGeo<D, DT, MT>;
    using X = Mma<DT>;
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t sbase = smem_u32(smem);
    unsigned long long* smask = reinterpret_cast<unsigned long long*>(smem + G::OFF_MASK);
    float2* sml = reinterpret_cast<float2*>(smem + G::OFF_ML);
    float* sscale = reinterpret_cast<float*>(smem + G::OFF_SCALE);
    long long* sscan = reinterpret_cast<long long*>(smem + G::OFF_SCAN);

    const bool blocks = P.idx != nullptr;
    const int upb = (blocks ? P.T : 1) * P.H * P.mtiles;  // units of a sequence
    AttendShare sh = attend_share<G::NT>(P, upb, sscan);
    if (blocks) asm volatile("griddepcontrol.wait;" ::: "memory");  // the choice

    while (sh.pos < sh.end) {
        const AttendSeq seq = attend_seq(P, sh.b, false);
        const AttendPart part_of = attend_part(P, sh, seq.tiles);
        const int u = part_of.u, tile0 = part_of.tile0, ntile = part_of.n;
        if (ntile == 0) {
            attend_advance(P, sh, part_of.step, seq.tiles, upb);
            continue;
        }
        const int mt = u % P.mtiles, h = (u / P.mtiles) % P.H, t0 = blocks ? u / P.mtiles / P.H : 0;
        const int mrows_all = blocks ? P.G : P.T * P.G;
        const int m0 = mt * G::MR, mrows = min(G::MR, mrows_all - m0);
        // rows this unit may see at all, the first drafted row, and the virtual rows of this share
        const int lim = seq.tokens == 0 ? 0 : blocks ? seq.len - (P.T - 1 - t0) : seq.len;
        const int base = seq.len - seq.tokens;
        const bool masked = !blocks && (P.mask != nullptr || seq.tokens > 1);
        const int32_t* bidx = blocks ? P.idx + (((long long)sh.b * P.T + t0) * P.H + h) * P.keep : nullptr;
        const int vrow0 = tile0 * kAttendTile;
        int vrows = ntile * kAttendTile;
        if (blocks)
            vrows = min(vrows, (P.keep << P.block_shift) - vrow0);
        else
            vrows = min(vrows, seq.len - vrow0);
        if (seq.tokens == 0) vrows = 0;
        const int nt16 = (max(vrows, 0) + kWarpRows - 1) / kWarpRows;

        // ---- this warp's tiles w, w + NW, ... ; the first are on their way before anything else
        __syncthreads();  // the ring holds nothing of the unit before
        const int mine = (nt16 - w + G::NW - 1) / G::NW;  // tiles of this warp (<= 0: none)
        // lane l: byte offset (-1: not there) and first row of this warp's tile 32 * (i / 32) + l, looked up
        // 32 tiles at a time so that the chain of table reads is not paid per tile
        long long off = -1, off_c = -1;
        int row_of = 0, row_c = 0;
        const uint32_t ring = sbase + w * G::STAGES * G::STAGE;
        auto issue = [&](int i) {
            if (i < mine) {
                if ((i & 31) == 0) {
                    off = -1;
                    row_of = 0x7fffffff;
                    if (i + lane < mine) {
                        const int v = vrow0 + (w + (i + lane) * G::NW) * kWarpRows;
                        int r = v;
                        if (blocks) {
                            const int j = __ldcg(bidx + (v >> P.block_shift));  // written while this kernel was starting
                            r = j < 0 ? 0x7fffffff : (j << P.block_shift) + (v & ((1 << P.block_shift) - 1));
                        }
                        row_of = r;
                        if (r < lim) off = attend_offset(P, sh.b, h, r);
                    }
                }
                const long long o = __shfl_sync(~0u, off, i & 31);
                const int r0 = __shfl_sync(~0u, row_of, i & 31);
                const int there = o < 0 ? 0 : lim - r0;  // rows that exist
                const uint32_t dst = ring + (i % G::STAGES) * G::STAGE;
                const uint8_t* k = P.K + (o < 0 ? 0 : o);
                const uint8_t* v = P.V + (o < 0 ? 0 : o);
#pragma unroll
                for (int j = 0; j < kWarpRows * G::CPR / 32; ++j) {
                    const int id = j * 32 + lane, r = id / G::CPR, c = id % G::CPR;
                    const bool ok = r < there;
                    const long long src = ok ? (long long)r * P.ss + c * 16 : 0;
                    cp_async16(dst + r * G::PITCH + c * 16, k + src, ok);
                    cp_async16(dst + G::TENSOR + r * G::PITCH + c * 16, v + src, ok);
                }
            }
            cp_async_commit();
        };
#pragma unroll 1
        for (int i = 0; i < G::STAGES - 1; ++i) issue(i);
        // queries, masks and row scales of the unit
        {
            constexpr int PER = G::NT / G::MR;  // threads per query row
            const int m = tid / PER, part = tid % PER;
            const int row = m0 + m, t = t0 + row / P.G, g = row % P.G;
            const bool there = m < mrows;
            const uint16_t* q = P.Q + (long long)sh.b * P.q_sb + (long long)t * P.q_st + (long long)(h * P.G + g) * P.q_sh;
            float f = 1.f;
            if (DT == 2) {  // largest magnitude to [2^8, 2^9)
                float top = 0.f;
                if (there)
                    for (int d = part; d < D; d += PER) top = fmaxf(top, fabsf(Elem<0>::lo(__ldg(q + d))));
#pragma unroll
                for (int o = PER / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
                const int e = (__float_as_int(top) >> 23) & 255;
                // e = 0: zero or subnormal, e = 255: not finite
                if (e > 0 && e < 255) f = __int_as_float(min(262 - e, 254) << 23);
            }
            for (int d = part * 2; d < D; d += PER * 2) {
                uint32_t v = there ? __ldg(reinterpret_cast<const uint32_t*>(q + d)) : 0u;
                int at = d;
                if (DT == 2) {
                    v = MmaHalf::pack(Elem<0>::lo(v) * f, Elem<0>::hi(v) * f);
                    // the order of the channels in which a word of four fp8 values meets the fragments
                    const int c = (d & 15) >> 2, i = (d & 3) >> 1;
                    at = (d & ~15) + 2 * c + 8 * i;
                }
                *reinterpret_cast<uint32_t*>(smem + G::OFF_Q + m * G::QPITCH + at * 2) = v;
            }
            if (part == 0) {
                sscale[m] = P.scale_log2 / f;
                unsigned long long bits = 0;
                if (there && masked && t < seq.tokens)
                    bits = P.mask ? P.mask[(long long)sh.b * P.T + t] : (t == 63 ? ~0ull : (2ull << t) - 1);
                smask[m] = bits;
            }
        }
        __syncthreads();

        float acc[MT][D / 8][4], ref[MT][2], sum[MT][2], scl[MT][2];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][n][e] = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                ref[i][e] = -INFINITY;
                sum[i][e] = 0.f;
                scl[i][e] = sscale[i * 16 + (lane >> 2) + 8 * e];
            }
        }
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
            issue(i + G::STAGES - 1);
            if ((i & 31) == 0) {  // issue() is still inside this group of 32 tiles
                off_c = off;
                row_c = row_of;
            }
            cp_async_wait<G::STAGES - 1>();
            __syncwarp();
            const int r0 = __shfl_sync(~0u, row_c, i & 31);
            const long long ro = __shfl_sync(~0u, off_c, i & 31);
            const int there = ro < 0 ? 0 : min(kWarpRows, lim - r0);
            const uint32_t tk = ring + (i % G::STAGES) * G::STAGE, tv = tk + G::TENSOR;

            // S = Q K^T: two groups of eight rows
            float s[MT][2][4];
#pragma unroll
            for (int a = 0; a < MT; ++a)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[a][n][e] = 0.f;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                uint32_t kb[4];
                if (DT != 2) {
                    ldsm4(kb, tk + ((lane & 7) + ((lane >> 4) & 1) * 8) * G::PITCH + (ks * 2 + ((lane >> 3) & 1)) * 16);
                } else {
                    // 16 rows x 16 bytes: one word of four channels per row group and lane
                    uint32_t b0, b1;
                    asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0, %1}, [%2];"
                                 : "=r"(b0), "=r"(b1)
                                 : "r"(tk + (lane & 15) * G::PITCH + ks * 16)
                                 : "memory");
                    uint32_t p0[2], p1[2];
                    Elem<2>::expand(b0, p0);
                    Elem<2>::expand(b1, p1);
                    kb[0] = p0[0];
                    kb[1] = p0[1];
                    kb[2] = p1[0];
                    kb[3] = p1[1];
                }
#pragma unroll
                for (int a = 0; a < MT; ++a) {
                    uint32_t qa[4];
                    ldsm4(qa, sbase + G::OFF_Q + (a * 16 + (lane & 15)) * G::QPITCH + (ks * 2 + (lane >> 4)) * 16);
                    X::mma(s[a][0], qa, kb[0], kb[1]);
                    X::mma(s[a][1], qa, kb[2], kb[3]);
                }
            }

            // softmax step
            const bool some_hidden = there < kWarpRows || (masked && r0 + kWarpRows > base);
            uint32_t pa[MT][4];
#pragma unroll
            for (int a = 0; a < MT; ++a) {
                float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = s[a][n][e] * scl[a][e >> 1];
                        if (some_hidden) {
                            const int c = n * 8 + (lane & 3) * 2 + (e & 1), j = r0 + c - base;
                            bool see = c < there;
                            if (masked && j >= 0)
                                see = see && ((smask[a * 16 + (lane >> 2) + 8 * (e >> 1)] >> (j & 63)) & 1);
                            x = see ? x : -INFINITY;
                        }
                        s[a][n][e] = x;
                        top[e >> 1] = fmaxf(top[e >> 1], x);
                    }
                bool grew = false;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[e] = fmaxf(top[e], __shfl_xor_sync(~0u, top[e], 1));
                    top[e] = fmaxf(top[e], __shfl_xor_sync(~0u, top[e], 2));
                    top[e] -= X::kRefShift;
                    grew |= top[e] > ref[a][e];
                }
                if (__any_sync(~0u, grew)) {
                    float f[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float r = fmaxf(ref[a][e], top[e]);
                        f[e] = r == -INFINITY ? 1.f : ex2(ref[a][e] - r);
                        ref[a][e] = r;
                        sum[a][e] *= f[e];
                    }
#pragma unroll
                    for (int n = 0; n < D / 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[a][n][e] *= f[e >> 1];
                }
                float at[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) at[e] = ref[a][e] == -INFINITY ? 0.f : ref[a][e];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[a][n][e] = ex2(s[a][n][e] - at[e >> 1]);
                        sum[a][e >> 1] += s[a][n][e];
                    }
                pa[a][0] = X::pack(s[a][0][0], s[a][0][1]);
                pa[a][1] = X::pack(s[a][0][2], s[a][0][3]);
                pa[a][2] = X::pack(s[a][1][0], s[a][1][1]);
                pa[a][3] = X::pack(s[a][1][2], s[a][1][3]);
            }

            // A drafted row hidden from some tokens must not reach them through 0 * inf: rows with
            // values that are not finite leave the tile and are added to the tokens that see them.
            if (masked && r0 + kWarpRows > base) {
                const unsigned char* vt = smem + (tv - sbase);
                for (int r = max(0, base - r0); r < there; ++r) {
                    bool odd = false;
                    for (int c = lane; c < G::ROWB / 4; c += 32) {
                        const uint32_t v = *reinterpret_cast<const uint32_t*>(vt + r * G::PITCH + c * 4);
                        if (DT == 0) odd |= (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
                        if (DT == 1) odd |= (v & 0x7c00u) == 0x7c00u || (v & 0x7c000000u) == 0x7c000000u;
                        if (DT == 2)
                            for (int e = 0; e < 4; ++e) odd |= ((v >> (8 * e)) & 0x7f) == 0x7f;
                    }
                    if (!__any_sync(~0u, odd)) continue;
#pragma unroll
                    for (int a = 0; a < MT; ++a)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            // probability of row r for query row (lane >> 2) + 8 e, from the lane that holds it
                            const int src = (lane & ~3) | ((r & 7) >> 1);
                            const float p0 = __shfl_sync(~0u, r < 8 ? s[a][0][2 * e] : s[a][1][2 * e], src);
                            const float p1 = __shfl_sync(~0u, r < 8 ? s[a][0][2 * e + 1] : s[a][1][2 * e + 1], src);
                            const float p = (r & 1) ? p1 : p0;
                            const bool see = (smask[a * 16 + (lane >> 2) + 8 * e] >> ((r0 + r - base) & 63)) & 1;
                            if (see) {
#pragma unroll
                                for (int n = 0; n < D / 8; ++n)
#pragma unroll
                                    for (int f = 0; f < 2; ++f) {
                                        const int d = DT == 2 ? (n >> 1) * 16 + (lane & 3) * 4 + 2 * f + (n & 1)
                                                              : n * 8 + (lane & 3) * 2 + f;
                                        float v;
                                        if (DT == 2) {
                                            uint32_t pr[2];
                                            Elem<2>::expand(vt[r * G::PITCH + d], pr);
                                            v = Elem<1>::lo(pr[0]);
                                        } else {
                                            v = q_to_float(*reinterpret_cast<const uint16_t*>(vt + r * G::PITCH + d * 2), DT == 1);
                                        }
                                        acc[a][n][2 * e + f] += p * v;
                                    }
                            }
                        }
                    __syncwarp();
                    for (int c = lane; c < G::ROWB / 4; c += 32)
                        *reinterpret_cast<uint32_t*>(smem + (tv - sbase) + r * G::PITCH + c * 4) = 0u;
                    __syncwarp();
                }
            }

            // O += P V
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
                uint32_t vb[4];
                if (DT != 2) {
                    ldsm4_t(vb, tv + (lane & 15) * G::PITCH + (n * 2 + (lane >> 4)) * 16);
                } else {
                    // two bytes (channels 2c, 2c + 1) of two rows per lane: rows become the pairs
                    uint32_t b0, b1;
                    asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0, %1}, [%2];"
                                 : "=r"(b0), "=r"(b1)
                                 : "r"(tv + (lane & 15) * G::PITCH + n * 16)
                                 : "memory");
                    uint32_t p0[2], p1[2];
                    Elem<2>::expand(__byte_perm(b0, 0, 0x3120), p0);
                    Elem<2>::expand(__byte_perm(b1, 0, 0x3120), p1);
                    vb[0] = p0[0];
                    vb[1] = p1[0];
                    vb[2] = p0[1];
                    vb[3] = p1[1];
                }
#pragma unroll
                for (int a = 0; a < MT; ++a) {
                    X::mma(acc[a][2 * n], pa[a], vb[0], vb[1]);
                    X::mma(acc[a][2 * n + 1], pa[a], vb[2], vb[3]);
                }
            }
            __syncwarp();
        }
        cp_async_wait<0>();
        __syncthreads();  // the rings are idle: the warps' accumulators go there

        float* epi = reinterpret_cast<float*>(smem) + w * G::MR * (D + 4);
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                sum[a][e] += __shfl_xor_sync(~0u, sum[a][e], 1);
                sum[a][e] += __shfl_xor_sync(~0u, sum[a][e], 2);
                const int m = a * 16 + (lane >> 2) + 8 * e;
                if ((lane & 3) == 0) sml[w * G::MR + m] = make_float2(ref[a][e], sum[a][e]);
#pragma unroll
                for (int n = 0; n < D / 8; ++n)
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        const int d = DT == 2 ? (n >> 1) * 16 + (lane & 3) * 4 + 2 * f + (n & 1) : n * 8 + (lane & 3) * 2 + f;
                        epi[m * (D + 4) + d] = acc[a][n][2 * e + f];
                    }
            }
        __syncthreads();

        // who shares this unit: CTAs c0 .. c1
        const long long c0 = part_of.c0, c1 = part_of.c1;
        constexpr int PSIZE = G::MR * (D + 2);
        float* part = P.partials + (2ll * blockIdx.x + (c0 == (long long)blockIdx.x ? 1 : 0)) * PSIZE;
        for (int i = tid; i < mrows * (D / 4); i += G::NT) {
            const int m = i / (D / 4), d = (i % (D / 4)) * 4;
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < G::NW; ++k) top = fmaxf(top, sml[k * G::MR + m].x);
            float o[4] = {0.f, 0.f, 0.f, 0.f}, total = 0.f;
#pragma unroll
            for (int k = 0; k < G::NW; ++k) {
                const float2 ml = sml[k * G::MR + m];
                const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
                if (f == 0.f && ml.y == 0.f) continue;
                total += ml.y * f;
                const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<float*>(smem) + (k * G::MR + m) * (D + 4) + d);
                o[0] += v.x * f;
                o[1] += v.y * f;
                o[2] += v.z * f;
                o[3] += v.w * f;
            }
            if (c0 == c1) {
                attend_write<D, DT>(P, sh.b, h, t0, m0, seq.tokens, m, d, o, top, total);
            } else {
                __stcg(reinterpret_cast<float4*>(part + m * D + d), make_float4(o[0], o[1], o[2], o[3]));
                if (d == 0) __stcg(reinterpret_cast<float2*>(part + G::MR * D + 2 * m), make_float2(top, total));
            }
        }
        // who shares the unit, for the kernel that joins the partials: said once, by the CTA that starts it
        if (tid == 0 && c0 == (long long)blockIdx.x) P.shared[(long long)sh.b * upb + u] = make_int2(int(c0), int(c1));
        attend_advance(P, sh, part_of.step, seq.tiles, upb);
    }
}

// Joins the partials of shared units, in the order of their rows: a warp per query row, with the weights of up to
// 32 partials worked out first, one per lane, so that their reads do not wait for one another.  (The last CTA to
// arrive joined them at first: a CTA and 37 partials of 16 rows took 20 us.)
constexpr int kMergeWarps = 4;
template <int D, int MR, class Write>
__device__ __forceinline__ void attend_merge(const AttendParams& P, Write&& write) {
    constexpr int PSIZE = MR * (D + 2);
    constexpr int LANES = D / 4 < 32 ? D / 4 : 32;     // lanes of a row
    constexpr int SPLIT = D == 64 ? 2 : 1;             // partials at a time
    constexpr int N = D / LANES, BATCH = 8;            // channels of a lane, reads in flight
    const bool blocks = P.idx != nullptr;
    const int upb = (blocks ? P.T : 1) * P.H * P.mtiles, rows_all = blocks ? P.G : P.T * P.G;
    const int lane = threadIdx.x & 31, groups = (min(MR, rows_all) + kMergeWarps - 1) / kMergeWarps;
    const long long unit = blockIdx.x / groups;
    const int b = int(unit / upb), u = int(unit % upb), h = u / P.mtiles % P.H, t0 = blocks ? u / P.mtiles / P.H : 0;
    const int m0 = u % P.mtiles * MR, m = int(blockIdx.x % groups) * kMergeWarps + (threadIdx.x >> 5);
    const AttendSeq seq = attend_seq(P, b, false);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the partials
    const int2 who = __ldcg(P.shared + unit);
    if (who.x < 0 || who.x >= who.y || who.y >= P.ctas || m >= min(MR, rows_all - m0)) return;
    const int part = lane / LANES, d = lane % LANES * N;
    float top = -INFINITY, total = 0.f, o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.f;
    for (int first = who.x; first <= who.y; first += 32) {
        auto at = [&](int c) { return P.partials + (2ll * c + (c == who.x ? 1 : 0)) * PSIZE; };
        const int n = min(32, who.y - first + 1);
        float2 ml = make_float2(-INFINITY, 0.f);
        if (lane < n) ml = __ldcg(reinterpret_cast<const float2*>(at(first + lane) + MR * D + 2 * m));
        float r = ml.x;
#pragma unroll
        for (int s = 16; s; s >>= 1) r = fmaxf(r, __shfl_xor_sync(~0u, r, s));
        r = fmaxf(r, top);
        // a partial without rows weighs nothing; one whose sum is NaN has to stay
        const float weight = ml.x == -INFINITY && ml.y == 0.f ? 0.f : ex2(ml.x - r), back = top == -INFINITY ? 0.f : ex2(top - r);
        float sum = weight == 0.f && ml.y == 0.f ? 0.f : ml.y * weight;
#pragma unroll
        for (int s = 16; s; s >>= 1) sum += __shfl_xor_sync(~0u, sum, s);
        total = (top == -INFINITY ? 0.f : total * back) + sum;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = top == -INFINITY ? 0.f : o[i] * back;
        top = r;
        const uint32_t there = __ballot_sync(~0u, !(ml.x == -INFINITY && ml.y == 0.f));
        for (int c = 0; c < n; c += BATCH * SPLIT) {
            float4 v[BATCH][N / 4];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int x = c + k * SPLIT + part;
#pragma unroll
                for (int i = 0; i < N / 4; ++i)
                    v[k][i] = x < n && part < SPLIT ? __ldcg(reinterpret_cast<const float4*>(at(first + x) + m * D + d) + i) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int x = c + k * SPLIT + part;
                const float f = __shfl_sync(~0u, weight, x & 31);
                if (x >= n || part >= SPLIT || !(there >> x & 1)) continue;
#pragma unroll
                for (int i = 0; i < N / 4; ++i) {
                    o[4 * i] = fmaf(v[k][i].x, f, o[4 * i]);
                    o[4 * i + 1] = fmaf(v[k][i].y, f, o[4 * i + 1]);
                    o[4 * i + 2] = fmaf(v[k][i].z, f, o[4 * i + 2]);
                    o[4 * i + 3] = fmaf(v[k][i].w, f, o[4 * i + 3]);
                }
            }
        }
    }
    if constexpr (SPLIT == 2) {
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] += __shfl_xor_sync(~0u, o[i], 16);
    }
    if (part == 0) write(b, h, t0, m0, seq.tokens, m, d, o, top, total);
}
template <int D, int DT, int MT>
__global__ void __launch_bounds__(kMergeWarps * 32, 4)  // without the 4: 32 registers, hardly a read in flight, 1-3 us more
lagkv_attend_merge_kernel(const __grid_constant__ AttendParams P) {
    attend_merge<D, AttendGeo<D, DT, MT>::MR>(P, [&](int b, int h, int t0, int m0, int tokens, int m, int d, const auto& o, float top, float total) {
        attend_write<D, DT>(P, b, h, t0, m0, tokens, m, d, o, top, total);
    });
}

}  // namespace lagkv
