// Attention over the cache for many query rows (wide trees) -- 5th-generation tensor cores.
//
// The same mathematics and the same shares of the work as lagkv_attend_kernel.  With 33 or more query rows
// per KV head the products of a 128-row tile outgrow mma.sync (that kernel reached 150 TFLOP/s); here they
// run as tcgen05.mma with M = 128 query rows, accumulators and probabilities in tensor memory:
//     S[128 x 128] = Q K^T (both from shared memory),   O[128 x D] += P V (P from tensor memory).
// Two streams keep the tensor cores busy while the other one's softmax runs: with up to 128 query rows the
// streams take every other tile of rows and are joined at the end, with up to 256 each has its own 128
// query rows and both read the same tiles.
// Warps: 0-3 and 4-7 the softmax of stream 0 and 1 (a thread owns a query row); 8 issues the products; 9
// fetches tiles by TMA into swizzled shared memory, a box per page and 64 channels (the same tiles as cp.async
// cost three warps 10000 cycles a step, five times what the products take); the others help: they load the
// next unit's queries, mend V tiles -- rows behind the last one and hidden rows that are not finite become
// zeros, so that 0 * inf never happens -- and widen fp8 tiles, which land as they are, to fp16.
// Partials of shared units are 66 KB for 128 query rows.
// What it is near: at 128 rows and 16-bit caches HBM (16 x 8 x 9728 rows of 128 bf16 channels under 32 tokens of 4
// heads in 102 us: 64 % of the DRAM's peak, tensor cores 35 %).  At 256 rows no unit is full (2 x 8 x 131072 fp16 rows
// under 64 tokens in 270 us, tensor cores 49 %): of some 5200 cycles a step the products need 2850 and the 2 x 16384
// exponentials, 16 a cycle, 2050 beside them; the rest is the softmax warps, two to a scheduler, waiting for one
// part of their scores after the other.  fp8 caches: the way of a tile through shared memory, landed, widened and
// multiplied, with three slots for widened tiles at 128 and 96 channels and a place to land in for each group of helpers (8 x 8 x
// 19968 rows under 13 tokens in 123 us where HBM takes 41).
#pragma once
#include <cuda.h>

#include "lagkv_attend_kernels.cuh"

namespace lagkv {

constexpr int kWideTile = 128;        // rows of K and V per step
constexpr int kWideLead = 6;          // P.lead: 32 tokens over 16 x 9728 rows in 101 us, 108 with equal shares
constexpr int kWideRowFlags = 32;     // loads whose missing rows are remembered: more than the rings hold

template <int D_, int DT_, int MT_>
struct WideGeo {
    static constexpr int D = D_, DT = DT_, MT = MT_;  // MT = 1: streams split the rows, 2: the query rows
    static constexpr int EB = Elem<DT_>::EB;
    static constexpr int ROWB = D * EB, CPR = ROWB / 16;
    static constexpr int PANELS = (D + 63) / 64;       // 64 channels of 16 bits: 128-byte rows, swizzled
    static constexpr int PANEL = kWideTile * 128;
    static constexpr int SLOT = PANELS * PANEL;
    static constexpr int EXCH = 64 * kWideTile * 4;    // MT = 1: 32 channels of each stream's O for the other
    static constexpr int QBYTES = MT == 2 ? 2 * SLOT : SLOT + EXCH;
    static constexpr int WARPS = DT_ == 2 ? 16 : 12;   // more would leave the softmax too few registers
    static constexpr int NT = WARPS * 32;
    // Warps 10 ..: load queries; mend V tiles (16-bit), or widen tiles in groups, each every GROUPS-th tile
    static constexpr int HELP_WARPS = WARPS - 10, GROUPS = DT_ == 2 ? 3 : 1, HELP = HELP_WARPS / GROUPS * 32;
    // fp8: rows of a pass of a group, and the threads it takes; eight rows on the swizzle is the same again
    static constexpr int PASS = HELP / CPR & ~7, PASS_THREADS = PASS * CPR;
    static constexpr int MISC = 1024;
    static constexpr int RAW = DT_ == 2 ? kWideTile * ROWB : 0;  // an fp8 tile as it is stored ...
    // ... and how many are in flight: one or two for each group of helpers, which takes its own in turn.  A place that groups took in
    // turns could be waited for by a group one lap ahead of a copy that is late, and a parity does not tell that lap from the one before.
    // Two at 64 channels, where all eight slots still fit: 16 x 8 x 8192 rows under 64 query rows 86.5 us, 93.5 with one, 8 x 8 x 16384
    // under 256 query rows 110.4 and 109.2, so one there.
    static constexpr int RS = DT_ != 2 ? 0 : D_ == 64 && MT_ == 1 ? 2 * GROUPS : GROUPS;
    static constexpr int NS_FIT = (232448 - 1024 - MISC - QBYTES - RS * RAW) / SLOT;
    static constexpr int NS = NS_FIT > 8 ? 8 : NS_FIT;           // tiles of K or V in the ring
    static constexpr int CHUNKS = kWideTile * CPR;               // 16-byte pieces of a stored tile
    static constexpr int SMEM = 1024 + QBYTES + NS * SLOT + RS * RAW + MISC;
    static constexpr int PSIZE = MT * kWideTile * (D + 2);
    static_assert(NS >= 3, "a released tile may need the two behind it");
    static_assert(D <= 128 && D % 32 == 0, "tensor memory: 2 x 128 columns of S, 2 x D of O");
};

// ---- tcgen05
__device__ __forceinline__ void tm_alloc(uint32_t smem_dst) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_dst) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tm_free(uint32_t base) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(base) : "memory");
}
__device__ __forceinline__ void tm_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tm_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// High word of the shared memory operands: rows in groups of eight (1024 bytes), swizzled by 128 bytes.
constexpr uint32_t kDescHi = 1024u >> 4 | 1u << 14 | 2u << 29;
// Issued by the lane whose `lead` is set, in code that the whole warp runs: operands that are the same in all
// lanes stay in uniform registers, moving them there one by one cost more than the products.
__device__ __forceinline__ void mma_ss(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 q, %6, 0;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\t"
        "mov.b64 b, {%2, %5};\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"(kDescHi), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc) {  // adds to d
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 b;\n\tsetp.ne.b32 q, %6, 0;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(1), "n"(kDescHi), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void tm_commit(uint32_t lead, uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
        "r"(lead)
        : "memory");
}
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}
__device__ __forceinline__ void tm_ld32(uint32_t (&r)[32], uint32_t a) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(a)
        : "memory");
}
__device__ __forceinline__ void tm_st32(uint32_t a, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(a),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t a, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16};" ::"r"(a),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ uint32_t tm_read1(uint32_t a) {  // one column, waited for
    uint32_t r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=r"(r) : "r"(a) : "memory");
    return r;
}
// waits for this thread's loads from tensor memory; `r` is named so that nothing reads it earlier
__device__ __forceinline__ void tm_wait_ld(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Low word of a shared memory operand.  `lead`: bytes between panels of 64 channels (read when the panels run
// along the operand's outer dimension, as in V).
__device__ __forceinline__ uint32_t smem_desc_lo(uint32_t addr, uint32_t lead) { return (addr & 0x3ffff) >> 4 | lead >> 4 << 16; }
// Instruction word of kind::f16: fp32 accumulators, M = 128.
__device__ __forceinline__ constexpr uint32_t mma_idesc(bool bf16, bool b_rows_are_k, int n) {
    return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (b_rows_are_k ? 1u << 16 : 0u) | uint32_t(n / 8) << 17 | uint32_t(128 / 16) << 24;
}

// Place of the K tile and of the V tile of step i in a unit's sequence of loads (n steps).  Streams that
// split the rows need the scores of two steps before the first V: K runs one step ahead.
template <int MT>
__device__ __forceinline__ int load_of_k(int i) { return MT == 2 ? 2 * i : i == 0 ? 0 : 2 * i - 1; }
template <int MT>
__device__ __forceinline__ int load_of_v(int i, int n) { return MT == 2 ? 2 * i + 1 : 2 * i + 1 + (i + 1 < n); }

// The unit at a CTA's position, as every role sees it.
struct WideUnit {
    AttendSeq seq;
    int u, h, m0, mrows, tile0, n;  // n: steps of this share
    int step, first_cta, last_cta;
    int lim, base;                  // rows seen at all, first drafted row
    bool masked;
};
template <class G>
__device__ __forceinline__ WideUnit wide_unit(const AttendParams& P, const AttendShare& sh) {
    WideUnit w;
    w.seq = attend_seq<kWideTile>(P, sh.b, false);
    const AttendPart a = attend_part(P, sh, w.seq.tiles);
    w.u = a.u;
    w.tile0 = a.tile0;
    w.n = a.n;
    w.step = a.step;
    w.first_cta = int(a.c0);
    w.last_cta = int(a.c1);
    w.h = w.u / P.mtiles % P.H;
    w.m0 = w.u % P.mtiles * (G::MT * kWideTile);
    w.mrows = min(G::MT * kWideTile, P.T * P.G - w.m0);
    w.lim = w.seq.tokens == 0 ? 0 : w.seq.len;
    w.base = w.seq.len - w.seq.tokens;
    w.masked = P.mask != nullptr || w.seq.tokens > 1;
    return w;
}
// Goes on to the next unit with rows (`w` is the present one, or any when n == 0); false: none.
template <class G>
__device__ __forceinline__ bool wide_next(const AttendParams& P, AttendShare& sh, WideUnit& w, int units_per_seq) {
    do {
        attend_advance(P, sh, w.step, w.seq.tiles, units_per_seq);
        if (sh.pos >= sh.end) return false;
        w = wide_unit<G>(P, sh);
    } while (w.n == 0);
    return true;
}
// The first unit with rows.
template <class G>
__device__ __forceinline__ bool wide_first(const AttendParams& P, AttendShare& sh, WideUnit& w, int units_per_seq) {
    if (sh.pos >= sh.end) return false;
    w = wide_unit<G>(P, sh);
    return w.n > 0 || wide_next<G>(P, sh, w, units_per_seq);
}

// fp8 caches: the power of two that brings a row of bf16 queries to [2^8, 2^9), and its largest magnitude.
__device__ __forceinline__ float query_factor(float top) {
    const int e = (__float_as_int(top) >> 23) & 255;  // 0: zero or subnormal, 255: not finite
    return e > 0 && e < 255 ? __int_as_float(min(262 - e, 254) << 23) : 1.f;
}
__device__ __forceinline__ float largest_of(const uint4& v) {
    const uint32_t x[4] = {v.x, v.y, v.z, v.w};
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, fmaxf(fabsf(Elem<0>::lo(x[k])), fabsf(Elem<0>::hi(x[k]))));
    return top;
}

// The queries of a unit into swizzled shared memory (`to`), 32 rows at a time by warp `warp` of `warps`: a lane
// finds its row's place once, all lanes copy.
template <class G>
__device__ __forceinline__ void load_queries(const AttendParams& P, const WideUnit& U, int b, unsigned char* to, int warp, int warps) {
    constexpr int D = G::D, CH = D / 8;  // 16-byte pieces of a row
    const int lane = threadIdx.x & 31;
    const uint16_t* q0 = P.Q + (long long)b * P.q_sb + (long long)(U.h * P.G) * P.q_sh;
    auto place = [&](int r, int ch) {
        return reinterpret_cast<uint4*>(to + (r >> 7) * G::SLOT + (ch >> 3) * G::PANEL + (r & 127) * 128 + (((ch & 7) ^ (r & 7)) << 4));
    };
#pragma unroll 1
    for (int r0 = warp * 32; r0 < G::MT * kWideTile; r0 += warps * 32) {
        const int row = U.m0 + r0 + lane;
        const long long off = r0 + lane < U.mrows ? (long long)(row / P.G) * P.q_st + (long long)(row % P.G) * P.q_sh : -1;
        if constexpr (G::DT != 2) {
#pragma unroll 4
            for (int k = 0; k < CH; ++k) {
                const int id = k * 32 + lane, r = r0 + id / CH, ch = id % CH;
                const long long o = __shfl_sync(~0u, off, id / CH);
                cp_async16(smem_u32(place(r, ch)), o >= 0 ? q0 + o + ch * 8 : P.Q, o >= 0);
            }
        } else {  // a lane takes its row whole and scales it
            uint4 v[CH];
            float top = 0.f;
#pragma unroll
            for (int ch = 0; ch < CH; ++ch) v[ch] = off >= 0 ? __ldg(reinterpret_cast<const uint4*>(q0 + off) + ch) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int ch = 0; ch < CH; ++ch) top = fmaxf(top, largest_of(v[ch]));
            const float f = query_factor(top);
#pragma unroll
            for (int ch = 0; ch < CH; ++ch) {
                uint32_t y[4] = {v[ch].x, v[ch].y, v[ch].z, v[ch].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = MmaHalf::pack(Elem<0>::lo(y[k]) * f, Elem<0>::hi(y[k]) * f);
                *place(r0 + lane, ch) = make_uint4(y[0], y[1], y[2], y[3]);
            }
        }
    }
    cp_async_commit();
    cp_async_wait<0>();
    fence_proxy_async();
}

// A walk over the loads of a CTA's share, in order.
template <class G>
struct WideCursor {
    AttendShare sh;
    WideUnit U;
    int l;       // load of the unit
    uint32_t c;  // loads before this one
    bool more;
    __device__ __forceinline__ void start(const AttendShare& s, const WideUnit& u, bool any) {
        sh = s;
        U = u;
        l = 0;
        c = 0;
        more = any;
    }
    __device__ __forceinline__ void next(const AttendParams& P, int units_per_seq) {
        ++c;
        if (++l == 2 * U.n) {
            l = 0;
            more = wide_next<G>(P, sh, U, units_per_seq);
        }
    }
    __device__ __forceinline__ bool is_v() const {
        return G::MT == 2 ? (l & 1) != 0 : l == 2 * U.n - 1 || (l >= 2 && !(l & 1));
    }
    __device__ __forceinline__ int row0() const {  // first row of the tile
        const int i = G::MT == 2 ? l >> 1 : is_v() ? (l == 2 * U.n - 1 ? U.n - 1 : l / 2 - 1) : (l + 1) >> 1;
        return (U.tile0 + i) * kWideTile;
    }
    // a V tile with rows that enter as zeros, or that may
    __device__ __forceinline__ bool mend(uint32_t missing) const { return missing || careful() || row0() + kWideTile > U.lim; }
    // drafted V rows that are not finite are kept out of the tile
    __device__ __forceinline__ bool careful() const { return U.masked && is_v() && row0() + kWideTile > U.base; }
};

template <int D, int DT, int MT>
__global__ void __launch_bounds__(WideGeo<D, DT, MT>::NT, 1)
lagkv_attend_wide_kernel(const __grid_constant__ AttendParams P, const __grid_constant__ CUtensorMap map_k,
                         const __grid_constant__ CUtensorMap map_v) {
    using G = WideGeo<D, DT, MT>;
    using X = Mma<DT>;
    extern __shared__ unsigned char raw[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, w = __shfl_sync(~0u, tid >> 5, 0);  // the same in all lanes, visibly
    const uint32_t sbase = (smem_u32(raw) + 1023u) & ~1023u;
    unsigned char* smem = raw + (sbase - smem_u32(raw));
    const uint32_t s_q = sbase, s_ring = sbase + G::QBYTES, s_raw = s_ring + G::NS * G::SLOT, s_misc = s_raw + G::RS * G::RAW;
    unsigned char* misc = smem + (s_misc - sbase);
    float* exch = reinterpret_cast<float*>(smem + G::SLOT);  // MT = 1
    // misc: barriers (tile ready, place free, landed but not ready; scores, probabilities twice, O; queries in
    // place, their place free), the rows of each V tile that are not finite, the missing 16-row groups of each
    // load, scheduling scratch, barriers (places to land in free)
    const uint32_t b_full = s_misc, b_empty = b_full + 8 * 8, b_land = b_empty + 8 * 8, b_raw_free = s_misc + 768, b_s = b_land + 8 * 8,
                   b_p = b_s + 16, b_p2 = b_p + 16, b_o = b_p2 + 16, b_q = b_o + 16, b_q_free = b_q + 8;
    uint32_t* odd_rows = reinterpret_cast<uint32_t*>(misc + 288);                     // [8][4]
    volatile uint32_t* gone = reinterpret_cast<volatile uint32_t*>(misc + 416);       // [kWideRowFlags]
    long long* scan = reinterpret_cast<long long*>(misc + 544);                       // [16 + 2]
    uint32_t* tm_slot = reinterpret_cast<uint32_t*>(misc + 704);
    // One warp does not get the boxes of a paged cache's tiles out in time: one of the two helping warps fetches the V
    // tiles (16 x 8 x 8192 bf16 rows under 16 tokens of 4 heads, pages of 16 / 32 / 64 rows: 104 / 102 / 102 us at 128
    // channels, 135 / 107 / 105 without; 64 channels 75 / 70 / 69, without 96 / 89 / 86).  fp8 tiles are half the boxes,
    // and their helpers have no time to give.
    const bool two = DT != 2 && P.block_table != nullptr;
    const int helpers = G::HELP_WARPS - two, help = DT == 2 ? G::HELP : helpers * 32;

    if (tid == 0) {
        for (int i = 0; i < G::NS; ++i) {
            mbar_init(b_full + 8 * i, 1);
            mbar_init(b_empty + 8 * i, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(b_s + 8 * s, 1);
            mbar_init(b_p + 8 * s, 4);
            mbar_init(b_p2 + 8 * s, 4);
            mbar_init(b_o + 8 * s, 1);
        }
        for (int i = 0; i < (DT == 2 ? G::RS : G::NS); ++i) mbar_init(b_land + 8 * i, 1);
        for (int i = 0; i < G::RS; ++i) mbar_init(b_raw_free + 8 * i, 1);
        mbar_init(b_q, helpers);
        mbar_init(b_q_free, 1);
        fence_mbar_init();
    }
    if (w == 8) {
        __syncwarp();
        tm_alloc(smem_u32(tm_slot));
        tm_fence_before();
    }
    const int upb = P.H * P.mtiles;
    AttendShare sh = attend_share<G::NT, kWideTile>(P, upb, scan);
    WideUnit U;
    bool any = wide_first<G>(P, sh, U, upb);
    if (any) load_queries<G>(P, U, sh.b, smem, w, G::WARPS);  // the first unit's, by all
    __syncthreads();
    tm_fence_after();
    const uint32_t tm = __shfl_sync(~0u, *reinterpret_cast<volatile uint32_t*>(tm_slot), 0);
    // tensor memory columns: S (and P over it) of stream 0, 1 at 0, 128; O at 256, 256 + D
    constexpr int kO = 256;
    bool ok = true;

    if (w == 9 || (two && w == 11)) {
        // ------------------------------------------------------------------ K and V tiles
        // The tile as boxes of the tensor map, a lane each: 64 channels (fp8: whole rows) of the rows of a
        // page.  Boxes behind the last row and pages outside the pool are left out.
        constexpr int BP = DT == 2 ? 1 : G::PANELS;
        const int box_rows = P.block_table == nullptr ? kWideTile : min(kWideTile, 1 << P.page_shift);
        const int box = lane / BP, panel = lane % BP;
        const uint32_t box_bytes = uint32_t(box_rows) * (DT == 2 ? G::ROWB : 128);
        WideCursor<G> at;
        at.start(sh, U, any);
        for (; at.more; at.next(P, upb)) {
            if (two && at.is_v() != (w == 11)) continue;
            const int row = at.row0() + box * box_rows;
            bool there = box < kWideTile / box_rows && row < at.U.lim;
            const bool wanted = there;
            int c1 = row, c3 = at.sh.b;
            if (there && P.block_table != nullptr) {
                c3 = __ldg(P.block_table + (long long)at.sh.b * P.max_blocks + (row >> P.page_shift));
                c1 = row & ((1 << P.page_shift) - 1);
                if (c3 < 0 || c3 >= P.num_pages) {
                    there = false;
                    record_status(P.status, ST_EINVAL, at.sh.b);
                }
            }
            const int boxes = __popc(__ballot_sync(~0u, there));
            const unsigned missing = __ballot_sync(~0u, wanted && !there && panel == 0);
            uint32_t flags = 0;  // a bit per group of 16 rows whose page is not in the pool
            for (unsigned m = missing; m; m &= m - 1) flags |= ((1u << box_rows / 16) - 1) << (__ffs(int(m)) - 1) / BP * box_rows / 16;
            const bool is_v = at.is_v();
            uint32_t dst, bar;
            bool free;
            if (DT == 2) {
                const uint32_t place = at.c % (G::RS ? G::RS : 1);
                free = int(at.c) < G::RS || mbar_wait_bounded(b_raw_free + 8 * place, (at.c / (G::RS ? G::RS : 1) + 1) & 1);
                dst = s_raw + place * G::RAW;
                bar = b_land + 8 * place;
            } else {
                const uint32_t slot = at.c % G::NS;
                free = at.c < uint32_t(G::NS) || mbar_wait_bounded(b_empty + 8 * slot, (at.c / G::NS + 1) & 1);
                dst = s_ring + slot * G::SLOT;
                bar = (is_v && at.mend(flags) ? b_land : b_full) + 8 * slot;
            }
            if (!free) {
                if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
                ok = false;
                break;
            }
            if (lane == 0) {
                gone[at.c % kWideRowFlags] = flags;
                mbar_arrive_expect_tx(bar, boxes * box_bytes);
            }
            __syncwarp();
            if (there)
                asm volatile(
                    "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
                        dst + panel * G::PANEL + box * box_bytes),
                    "l"(is_v ? &map_v : &map_k), "r"(panel * 64), "r"(c1), "r"(at.U.h), "r"(c3), "r"(bar)
                    : "memory");
        }
    } else if (w > 9) {
        // ------------------------------------------------------------------ help
        const int group = (w - 10) / (G::HELP / 32), ptid = tid - 10 * 32 - group * G::HELP;
        // after a wait that ran out the walk goes on to its end without waiting, so that the barrier among these
        // warps still matches
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (ok && !mbar_wait_bounded(bar, parity)) {
                if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
                ok = false;
            }
        };
        auto meet = [&]() { named_bar_sync(2 + group, help); };
        auto not_finite = [](const uint4& v) {
            const uint32_t x[4] = {v.x, v.y, v.z, v.w};
            bool odd = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (DT == 0) odd |= (x[k] & 0x7f80u) == 0x7f80u || (x[k] & 0x7f800000u) == 0x7f800000u;
                if (DT == 1) odd |= (x[k] & 0x7c00u) == 0x7c00u || (x[k] & 0x7c000000u) == 0x7c000000u;
                if (DT == 2)
                    for (int e = 0; e < 4; ++e) odd |= ((x[k] >> (8 * e)) & 0x7f) == 0x7f;
            }
            return odd;
        };
        // Notes the drafted rows of a V tile that are not finite; `piece(id)` gives 16 bytes of row id / CPR.  Rows of
        // `groups` have no page: nothing was loaded for them, their place holds what an older tile left there.
        auto note_odd = [&](const WideCursor<G>& x, int slot, uint32_t groups, auto&& piece) {
            if (ptid < 4) odd_rows[slot * 4 + ptid] = 0u;
            meet();
            const int first = max(0, x.U.base - x.row0()) * G::CPR, last = min(kWideTile, x.U.lim - x.row0()) * G::CPR;
#pragma unroll 4
            for (int id = first + ptid; id < last; id += help)
                if (!(groups >> (id / G::CPR >> 4) & 1) && not_finite(piece(id))) atomicOr(&odd_rows[slot * 4 + id / G::CPR / 32], 1u << (id / G::CPR & 31));
            meet();
        };
        // the groups of 16 rows of a V tile whose pages are not in the pool
        auto missing_groups = [&](const WideCursor<G>& x) -> uint32_t {
            if (P.block_table == nullptr) return 0u;
            const int row = x.row0() + 16 * (lane & 7);
            bool miss = false;
            if (row < x.U.lim) {
                const int page = __ldg(P.block_table + (long long)x.sh.b * P.max_blocks + (row >> P.page_shift));
                miss = page < 0 || page >= P.num_pages;
            }
            return __ballot_sync(~0u, miss) & 255u;
        };
        auto zero_row = [&](const WideCursor<G>& x, int slot, int r, uint32_t groups, bool careful) {
            return x.row0() + r >= x.U.lim || (groups >> (r >> 4) & 1) || (careful && (odd_rows[slot * 4 + (r >> 5)] >> (r & 31) & 1));
        };
        // where the rows that may have to be zeroed begin
        auto first_zero = [&](const WideCursor<G>& x, int slot, uint32_t groups, bool careful) {
            if (groups) return 0;
            const bool odd = careful && (odd_rows[slot * 4] | odd_rows[slot * 4 + 1] | odd_rows[slot * 4 + 2] | odd_rows[slot * 4 + 3]);
            return max(0, (odd ? min(x.U.base, x.U.lim) : x.U.lim) - x.row0());
        };
        uint32_t landed = 0, units = 0;  // parities of the places where tiles to mend land (16-bit); units behind
        // the load's turn among the groups, slot and place, and how often slots and places have been through
        int turn = 0, slot = 0, place = 0;
        uint32_t slot_lap = 0, place_lap = 0;
        WideCursor<G> at;
        at.start(sh, U, any);
        auto go_on = [&]() {
            if (G::GROUPS > 1 && ++turn == G::GROUPS) turn = 0;
            if (++slot == G::NS) slot = 0, ++slot_lap;
            if (DT == 2 && ++place == G::RS) place = 0, ++place_lap;
            at.next(P, upb);
        };
        for (; at.more; go_on()) {
            if (at.l == 0 && at.c > 0) {  // the next unit's queries, once the products with those before are done
                wait(b_q_free, units++ & 1);
                load_queries<G>(P, at.U, at.sh.b, smem, w - 10, helpers);
                __syncwarp();
                if (lane == 0 && ok) mbar_arrive(b_q);
            }
            if (DT == 2 ? turn != group : !at.is_v()) continue;
            uint32_t groups = 0;
            if (DT != 2) {
                groups = missing_groups(at);
                if (!at.mend(groups)) continue;
            }
            if (DT == 2) {
                wait(b_land + 8 * place, place_lap & 1);
            } else {
                wait(b_land + 8 * slot, landed >> slot & 1);
                landed ^= 1u << slot;
            }
            if (DT == 2 && at.is_v()) groups = gone[at.c % kWideRowFlags];
            // fp8: `groups` is what the fetching warp has left, which two warps of a group may read differently once a wait has run
            // out; whether they meet must not depend on it
            const bool mend = at.is_v() && at.mend(DT == 2 ? P.block_table != nullptr : groups), careful = at.careful();
            unsigned char* tile = smem + (s_ring - sbase) + slot * G::SLOT;
            auto piece = [&](int id) {
                constexpr int CPR16 = D / 8;
                const int r = id / CPR16, ch = id % CPR16;
                return reinterpret_cast<uint4*>(tile + (ch >> 3) * G::PANEL + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
            };
            if constexpr (DT == 2) {
                if (slot_lap > 0) wait(b_empty + 8 * slot, (slot_lap + 1) & 1);
                const unsigned char* from = smem + (s_raw - sbase) + place * G::RAW;
                if (careful) note_odd(at, slot, groups, [&](int id) { return *reinterpret_cast<const uint4*>(from + id * 16); });
                // A row's 16-byte pieces become two each.  Eight lanes store to one panel's halves of two rows: the
                // swizzle gives them all the banks.
                const int r = D == 128 ? (ptid >> 4) * 2 + (ptid >> 2 & 1) : ptid / G::CPR, ch = D == 128 ? (ptid >> 1 & 4) + (ptid & 3) : ptid % G::CPR;
                if (ptid < G::PASS_THREADS) {
                    from += r * G::ROWB + ch * 16;
                    unsigned char* to = tile + (ch >> 2) * G::PANEL + r * 128;
                    const int c0 = ((ch & 3) * 2 ^ (r & 7)) << 4, c1 = c0 ^ 16;
#pragma unroll 4
                    for (int i = 0; i < kWideTile / G::PASS; ++i) {
                        const uint4 x = *reinterpret_cast<const uint4*>(from + i * G::PASS * G::ROWB);
                        uint32_t a[2], b[2], e[2], f[2];
                        Elem<2>::expand(x.x, a);
                        Elem<2>::expand(x.y, b);
                        Elem<2>::expand(x.z, e);
                        Elem<2>::expand(x.w, f);
                        *reinterpret_cast<uint4*>(to + c0 + i * G::PASS * 128) = make_uint4(a[0], a[1], b[0], b[1]);
                        *reinterpret_cast<uint4*>(to + c1 + i * G::PASS * 128) = make_uint4(e[0], e[1], f[0], f[1]);
                    }
                }
                if (mend) meet();
            } else if (careful) {
                note_odd(at, slot, groups, [&](int id) { return *piece(id); });
            }
            if (mend)
                for (int id = first_zero(at, slot, groups, careful) * (D / 8) + ptid; id < kWideTile * (D / 8); id += help)
                    if (zero_row(at, slot, id / (D / 8), groups, careful)) *piece(id) = make_uint4(0u, 0u, 0u, 0u);
            fence_proxy_async();
            meet();
            if (ptid == 0 && ok) {
                mbar_arrive(b_full + 8 * slot);
                if (DT == 2) mbar_arrive(b_raw_free + 8 * place);
            }
        }
    } else if (w == 8) {
        // ------------------------------------------------------------------ the products
        constexpr uint32_t id_qk = mma_idesc(DT == 0, false, kWideTile), id_pv = mma_idesc(DT == 0, true, D);
        const uint32_t lead = elect_one();
        uint32_t slot = G::NS - 1, phase = 1;   // the load taken last (loads are taken in their order)
        uint32_t np = 0, nq = 0;                // parities of the streams' probabilities (a bit each), of units
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (!mbar_wait_bounded(bar, parity)) {
                if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
                ok = false;
            }
            return ok;
        };
        auto next_load = [&]() {
            if (++slot == uint32_t(G::NS)) {
                slot = 0;
                phase ^= 1;
            }
            return wait(b_full + 8 * slot, phase);
        };
        for (bool first = true; ok && any; first = false) {
            const int n = __shfl_sync(~0u, U.n, 0);
            if (!first) {  // the first unit's queries are there
                if (!wait(b_q, nq)) break;
                nq ^= 1;
            }
            // Step i: O += P V of step i and the scores of step i + LEAD, whose place the former has freed.
            constexpr int LEAD = MT == 2 ? 1 : 2;
#pragma unroll 1
            for (int i = -LEAD; i < n; ++i) {
                const bool has_v = i >= 0, has_k = i + LEAD < n;
                uint32_t v_slot = 0;
                if (has_v) {
                    if (!next_load()) break;
                    v_slot = slot;
                }
                if (has_k && !next_load()) break;
#pragma unroll 1
                for (int k = 0; k < MT; ++k) {
                    const int s = MT == 2 ? k : i & 1;
                    if (has_v) {
                        const uint32_t v = smem_desc_lo(s_ring + v_slot * G::SLOT, G::PANEL), parity = np >> s & 1;
                        np ^= 1u << s;
                        // the first 64 rows as soon as their probabilities are there, the others behind them
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            if (!wait((half ? b_p2 : b_p) + 8 * s, parity)) break;
                            tm_fence_after();
#pragma unroll
                            for (int ks = half * 4; ks < half * 4 + 4; ++ks)
                                mma_ts(lead, tm + kO + s * D, tm + s * 128 + ks * 8, v + ks * (2048 >> 4), id_pv);
                        }
                        if (!ok) break;
                    }
                    if (has_k) {
                        // addresses count in 16 bytes in the low word and never carry out of it
                        const uint32_t q = smem_desc_lo(s_q + (MT == 2 ? s * G::SLOT : 0), 16), kd = smem_desc_lo(s_ring + slot * G::SLOT, 16);
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks) {
                            const uint32_t o = ((ks >> 2) * G::PANEL + (ks & 3) * 32) >> 4;
                            mma_ss(lead, tm + s * 128, q + o, kd + o, id_qk, ks != 0);
                        }
                        tm_commit(lead, b_s + 8 * s);
                    } else if (has_v) {
                        tm_commit(lead, b_o + 8 * s);
                    }
                }
                if (!ok) break;
                if (has_v) tm_commit(lead, b_empty + 8 * v_slot);
                if (has_k) tm_commit(lead, b_empty + 8 * slot);
                if (i + LEAD == n - 1) tm_commit(lead, b_q_free);  // the unit's last scores
            }
            any = wide_next<G>(P, sh, U, upb);
        }
    } else {
        // ------------------------------------------------------------------ softmax of a stream
        const int s = w >> 2, m = tid & 127;
        const uint32_t lanes = uint32_t(w & 3) << 21;  // tensor memory lanes 32 (w % 4) ..
        const uint32_t t_s = tm + lanes + s * 128, t_o = tm + lanes + kO + s * D;
        uint32_t ns = 0, no = 0, c0 = 0;
        auto wait = [&](uint32_t bar, uint32_t parity) {
            // after a wait that ran out the barriers among these warps go on, everything else stops
            if (ok && !mbar_wait_bounded(bar, parity)) {
                if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
                ok = false;
            }
            tm_fence_after();
        };
        while (any) {
            const int mine = (MT == 2 ? U.n : (U.n - s + 1) / 2);  // steps of this stream
            const int mu = (MT == 2 ? s * kWideTile : 0) + m;      // this thread's query row in the unit
            const int row = U.m0 + mu, t = row / P.G;
            const bool there = mu < U.mrows;
            float f = 1.f;
            if (DT == 2 && there) {  // the factor that the row was stored with
                const uint16_t* q = P.Q + (long long)sh.b * P.q_sb + (long long)t * P.q_st + (long long)(U.h * P.G + row % P.G) * P.q_sh;
                float top = 0.f;
#pragma unroll 8
                for (int d = 0; d < D; d += 8) top = fmaxf(top, largest_of(__ldg(reinterpret_cast<const uint4*>(q + d))));
                f = query_factor(top);
            }
            // never 0, which would make NaN of the -infinity of hidden rows: below 2^-126 all logits (2^25 of it at most) are 0
            const float scl = DT == 2 ? fmaxf(P.scale_log2 / f, 0x1p-126f) : P.scale_log2;
            unsigned long long bits = 0;
            if (there && U.masked && t < U.seq.tokens)
                bits = P.mask ? P.mask[(long long)sh.b * P.T + t] : (t == 63 ? ~0ull : (2ull << t) - 1);
            // O starts at zero, every product adds to it
            {
                uint32_t z[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) z[k] = 0u;
#pragma unroll
                for (int d = 0; d < D; d += 32) tm_st32(t_o + d, z);
                tm_wait_st();
            }
            float ref = -INFINITY, sum = 0.f;
            for (int k = 0; k < mine; ++k) {
                const int i = MT == 2 ? k : 2 * k + s, r0 = (U.tile0 + i) * kWideTile;
                wait(b_s + 8 * s, ns++ & 1);
                const bool draft = U.masked && r0 + kWideTile > U.base;
                const uint32_t missing = gone[(c0 + load_of_k<MT>(i)) % kWideRowFlags];  // 16-row groups without a page
                const bool hidden = draft || missing || r0 + kWideTile > U.lim;
                // which of 32 rows from r on this query row sees
                auto seen32 = [&](int r) -> uint32_t {
                    uint32_t see = r >= U.lim ? 0u : U.lim - r >= 32 ? ~0u : (1u << (U.lim - r)) - 1;
                    if (missing >> ((r - r0) >> 4) & 1) see &= 0xffff0000u;
                    if (missing >> ((r - r0) >> 4) & 2) see &= 0x0000ffffu;
                    if (draft && r + 32 > U.base) {
                        const int j = r - U.base;  // drafted rows j ..
                        const uint32_t word = j >= 64 ? 0u : j >= 0 ? uint32_t(bits >> j) : (j > -32 ? uint32_t(bits << -j) | ((1u << -j) - 1) : ~0u);
                        see &= word;
                    }
                    return see;
                };
                // Two passes over the scores, the largest logit and then the probabilities (one pass that holds a
                // tile's probabilities until the largest is known spills and misses in the instruction cache).
                // The reference moves only when a probability would pass 2^6 of what it was set for: 120 us against 122.5
                // for 32 tokens, 312-317 against 326-332 for 64, where it moves with every larger logit.  In 64-bit
                // emulation (9728 rows of 128 channels) the rounding of P then costs 0.0017 of the output's norm instead of
                // 0.0012 in bf16, 0.00021 instead of 0.00015 in fp16: the largest probability is no longer exactly 1.
                uint32_t a[32], b[32], c[32];
                float top;
                if (!hidden) {
                    float t2[2] = {-INFINITY, -INFINITY};
                    auto largest = [&](const uint32_t (&x)[32]) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            t2[0] = fmaxf(t2[0], fmaxf(__uint_as_float(x[e]), __uint_as_float(x[e + 1])));
                            t2[1] = fmaxf(t2[1], fmaxf(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3])));
                        }
                    };
                    tm_ld32(a, t_s);
#pragma unroll 1
                    for (int q = 0; q < 128; q += 64) {
                        tm_wait_ld(a);
                        tm_ld32(b, t_s + q + 32);
                        largest(a);
                        tm_wait_ld(b);
                        if (q == 0) tm_ld32(a, t_s + 64);
                        largest(b);
                    }
                    top = fmaxf(t2[0], t2[1]);
                } else {
                    // logits that this query row does not see become -infinity in place
                    top = -INFINITY;
#pragma unroll 1
                    for (int q = 0; q < 4; ++q) {
                        tm_ld32(a, t_s + 32 * q);
                        const uint32_t see = seen32(r0 + 32 * q);
                        tm_wait_ld(a);
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            if (!(see >> e & 1)) a[e] = 0xff800000u;
                            top = fmaxf(top, __uint_as_float(a[e]));
                        }
                        tm_st32(t_s + 32 * q, a);
                    }
                    tm_wait_st();
                }
                top = top * scl - X::kRefShift;
                const bool first = ref == -INFINITY, grew = top > ref + 6.f || (first && top > -INFINITY);
                if (__any_sync(~0u, grew && !first)) {
                    const float g = grew && !first ? ex2(ref - top) : 1.f;
                    sum *= g;
#pragma unroll 1
                    for (int d = 0; d < D; d += 32) {
                        tm_ld32(a, t_o + d);
                        tm_wait_ld(a);
#pragma unroll
                        for (int e = 0; e < 32; ++e) a[e] = __float_as_uint(__uint_as_float(a[e]) * g);
                        tm_st32(t_o + d, a);
                    }
                    tm_wait_st();
                }
                if (grew) ref = top;
                const float at = ref == -INFINITY ? 0.f : ref;
                if (draft) {
                    // drafted rows that are not finite went into the tile as zeros: add them for those who see them
                    const uint32_t l = c0 + load_of_v<MT>(i, U.n);
                    wait(b_full + 8 * (l % G::NS), (l / G::NS) & 1);
#pragma unroll 1
                    for (int q = 0; q < 4; ++q) {
#pragma unroll 1
                        for (uint32_t odd = ok ? odd_rows[l % G::NS * 4 + q] : 0u; odd; odd &= odd - 1) {
                            const int e = __ffs(int(odd)) - 1, r = r0 + 32 * q + e;
                            const float z = __uint_as_float(tm_read1(t_s + 32 * q + e));
                            const bool see = seen32(r0 + 32 * q) >> e & 1;
                            const float p = see ? ex2(z * scl - at) : 0.f;
                            const long long off = attend_offset(P, sh.b, U.h, r & ~15);
                            if (off < 0) continue;  // no page: never noted
                            const uint8_t* v = P.V + off + (long long)(r & 15) * P.ss;
#pragma unroll 1
                            for (int d = 0; d < D; d += 32) {
                                tm_ld32(a, t_o + d);
                                tm_wait_ld(a);
#pragma unroll
                                for (int x = 0; x < 32; ++x) {
                                    float y;
                                    if (DT == 2) {
                                        uint32_t pr[2];
                                        Elem<2>::expand(__ldg(v + d + x), pr);
                                        y = Elem<1>::lo(pr[0]);
                                    } else {
                                        y = q_to_float(__ldg(reinterpret_cast<const uint16_t*>(v) + d + x), DT == 1);
                                    }
                                    if (see) a[x] = __float_as_uint(__uint_as_float(a[x]) + p * y);
                                }
                                tm_st32(t_o + d, a);
                                tm_wait_st();
                            }
                        }
                    }
                }
                // tells the issuing warp that 64 more columns of probabilities are in place
                auto hand_over = [&](uint32_t bar) {
                    tm_wait_st();
                    tm_fence_before();
                    __syncwarp();
                    if (lane == 0 && ok) mbar_arrive(bar + 8 * s);
                };
                {
                    const f32x2 scl2 = pack2(scl, scl), at2 = pack2(-at, -at);
                    f32x2 part[2] = {0ull, 0ull};
                    // Exponentials of 32 columns beside the sums and 16-bit forms of the 32 before them, written
                    // in turns: the special function unit takes eight cycles for what the others do in two.
                    auto raise = [&](uint32_t (&x)[32], int e) {
                        float p0, p1;
                        unpack2(fma2(pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), scl2, at2), p0, p1);
                        x[e] = __float_as_uint(ex2(p0));
                        x[e + 1] = __float_as_uint(ex2(p1));
                    };
                    auto finish = [&](const uint32_t (&x)[32], uint32_t (&p)[16], int e) {
                        const float p0 = __uint_as_float(x[e]), p1 = __uint_as_float(x[e + 1]);
                        part[e / 2 & 1] = add2(part[e / 2 & 1], pack2(p0, p1));
                        p[e / 2] = X::pack(p0, p1);
                    };
                    auto both = [&](uint32_t (&x)[32], const uint32_t (&before)[32], uint32_t to) {
                        uint32_t p[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            raise(x, e);
                            finish(before, p, e);
                        }
                        tm_st16(to, p);
                    };
                    tm_ld32(a, t_s);
                    tm_wait_ld(a);
                    tm_ld32(b, t_s + 32);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) raise(a, e);
                    tm_wait_ld(b);
                    tm_ld32(c, t_s + 64);
                    both(b, a, t_s);
                    tm_wait_ld(c);
                    tm_ld32(a, t_s + 96);
                    both(c, b, t_s + 16);
                    hand_over(b_p);
                    tm_wait_ld(a);
                    both(a, c, t_s + 32);
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) finish(a, p, e);
                    tm_st16(t_s + 48, p);
                    hand_over(b_p2);
                    float s0, s1;
                    unpack2(add2(part[0], part[1]), s0, s1);
                    sum += s0 + s1;
                }
            }
            if (mine > 0) wait(b_o + 8 * s, no++ & 1);

            // ---- the unit's result
            const int first_cta = U.first_cta, last_cta = U.last_cta;
            const bool shared = first_cta != last_cta;
            float* part = P.partials + (2ll * blockIdx.x + (first_cta == int(blockIdx.x) ? 1 : 0)) * G::PSIZE + (MT == 2 ? s * kWideTile * (D + 2) : 0);
            float mref = ref, msum = sum, f_own = 1.f;
            if (MT == 1) {  // both streams' references and sums; each finishes every other group of 32 channels
                float2* ml = reinterpret_cast<float2*>(exch);
                ml[s * kWideTile + m] = make_float2(ref, sum);
                named_bar_sync(1, 256);
                const float2 o = ml[(s ^ 1) * kWideTile + m];
                named_bar_sync(1, 256);
                mref = fmaxf(ref, o.x);
                f_own = ref == -INFINITY ? (sum == 0.f ? 0.f : 1.f) : ex2(ref - mref);
                const float f_other = o.x == -INFINITY ? (o.y == 0.f ? 0.f : 1.f) : ex2(o.x - mref);
                const float own = sum * f_own, other = o.y * f_other;
                msum = s == 0 ? own + other : other + own;
            }
            const bool writes = there && ok;
#pragma unroll 1
            for (int d0 = 0; d0 < D; d0 += MT == 1 ? 64 : 32) {
                uint32_t a[32];
                if (MT == 1) {
                    // hands over its part of the other's channels
                    const int give = d0 + 32 * (s ^ 1);
                    if (give < D) {
                        tm_ld32(a, t_o + give);
                        tm_wait_ld(a);
#pragma unroll
                        for (int e = 0; e < 32; ++e) exch[(s * 32 + e) * kWideTile + m] = __uint_as_float(a[e]) * f_own;
                    }
                    named_bar_sync(1, 256);
                }
                const int d = d0 + (MT == 1 ? 32 * s : 0);
                if (d < D) {
                    tm_ld32(a, t_o + d);
                    tm_wait_ld(a);
                    if (MT == 1) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            a[e] = __float_as_uint(__uint_as_float(a[e]) * f_own + exch[((s ^ 1) * 32 + e) * kWideTile + m]);
                    }
                    if (writes && shared) {  // channel by channel: a warp writes 32 rows side by side
#pragma unroll
                        for (int e = 0; e < 32; ++e) __stcg(part + (d + e) * kWideTile + m, __uint_as_float(a[e]));
                    } else if (writes) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            float o[8];
#pragma unroll
                            for (int x = 0; x < 8; ++x) o[x] = __uint_as_float(a[e + x]);
                            attend_write<D, DT>(P, sh.b, U.h, 0, U.m0, U.seq.tokens, mu, d + e, o, mref, msum);
                        }
                    }
                }
                if (MT == 1) named_bar_sync(1, 256);
            }
            if (shared && writes && (MT == 2 || s == 0)) __stcg(reinterpret_cast<float2*>(part + kWideTile * D + 2 * m), make_float2(mref, msum));
            // who shares the unit, for the kernel that joins the partials: said once, by the CTA that starts it
            if (tid == 0 && first_cta == int(blockIdx.x))
                P.shared[(long long)sh.b * upb + U.u] = ok ? make_int2(first_cta, last_cta) : make_int2(0, 0);
            c0 += 2 * U.n;
            any = wide_next<G>(P, sh, U, upb);
        }
    }
    tm_fence_before();
    // a wait that ran out may have left copies and products in flight: they get one more bounded chance
    if (__syncthreads_or(!ok)) {
        const unsigned long long t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 200000000ull) { /* bounded drain delay */ }
        __syncthreads();
    }
    if (w == 8) tm_free(tm);
}

// Joins the partials of shared units in the order of their rows: a CTA per 32 query rows of a unit, a lane
// per row, a warp per eighth of the channels.
constexpr int kJoinRows = 32, kJoinThreads = 256;
template <int D, int MT, class Write>
__device__ __forceinline__ void attend_join(const AttendParams& P, Write&& write) {
    constexpr int N = D / 8, PSIZE = MT * kWideTile * (D + 2);
    const int upb = P.H * P.mtiles, chunks = (min(MT * kWideTile, P.T * P.G) + kJoinRows - 1) / kJoinRows, chunk = blockIdx.x % chunks;
    const long long unit = blockIdx.x / chunks;
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the partials
    const int2 who = __ldcg(P.shared + unit);
    if (who.x < 0 || who.x >= who.y || who.y >= P.ctas) return;  // not shared (or, after a wait that gave up, not said)
    const int b = int(unit / upb), u = int(unit % upb), h = u / P.mtiles % P.H, m0 = u % P.mtiles * (MT * kWideTile);
    const int mu = chunk * kJoinRows + (threadIdx.x & 31), d0 = (threadIdx.x >> 5) * N;
    if (m0 + mu >= P.T * P.G) return;
    const AttendSeq seq = attend_seq<kWideTile>(P, b, false);
    const float* base = P.partials + mu / kWideTile * (kWideTile * (D + 2));
    const int m = mu % kWideTile;
    float top = -INFINITY, total = 0.f, o[N];
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = 0.f;
    constexpr int BATCH = 4;  // partials in flight
    for (int c = who.x; c <= who.y; c += BATCH) {
        float2 ml[BATCH];
        float v[BATCH][N];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const float* pp = base + (2ll * min(c + k, who.y) + (c + k == who.x ? 1 : 0)) * PSIZE;
            ml[k] = __ldcg(reinterpret_cast<const float2*>(pp + kWideTile * D + 2 * m));
#pragma unroll
            for (int d = 0; d < N; ++d) v[k][d] = __ldcg(pp + (d0 + d) * kWideTile + m);
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            if (c + k > who.y || (ml[k].x == -INFINITY && ml[k].y == 0.f)) continue;
            const float r = fmaxf(top, ml[k].x);
            const float fo = top == -INFINITY ? 0.f : ex2(top - r), fn = ex2(ml[k].x - r);
            total = total * fo + ml[k].y * fn;
#pragma unroll
            for (int d = 0; d < N; ++d) o[d] = o[d] * fo + v[k][d] * fn;
            top = r;
        }
    }
#pragma unroll
    for (int d = 0; d < N; d += 4) {
        const float x[4] = {o[d], o[d + 1], o[d + 2], o[d + 3]};
        write(b, h, m0, seq.tokens, mu, d0 + d, x, top, total);
    }
}
template <int D, int DT, int MT>
__global__ void __launch_bounds__(kJoinThreads)
lagkv_attend_join_kernel(const __grid_constant__ AttendParams P) {
    attend_join<D, MT>(P, [&](int b, int h, int m0, int tokens, int m, int d, const auto& o, float top, float total) {
        attend_write<D, DT>(P, b, h, 0, m0, tokens, m, d, o, top, total);
    });
}

}  // namespace lagkv
