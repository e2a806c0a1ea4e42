// Attention for many query rows over a cache held in 8 bits with block scales -- 5th-generation tensor cores.
//
// The shares of the work, the tiles by TMA, the helpers that widen them to fp16 in swizzled shared memory and the partials are those
// of lagkv_attend_wide_kernel; the mathematics of the scales is that of lagkv_attend_quant_kernel.  What differs:
// Each softmax stream (four warps, a thread owns a query row) takes items of 64 rows of a tile and has two places for
// their scores in tensor memory, so that the scores of its next item are there when it comes to them:
//     up to 128 query rows: stream s takes rows 64 s .. of every tile, both streams are joined at the end,
//     up to 256:            stream s has its own 128 query rows and takes both halves of every tile.
// 64 scores fit a thread's registers, and nothing spills with 512 threads.  Products wait for probabilities only, in the order of the
// items; a stream waits for the product of its item before when it hands over the next, long after that has ended, or
// before it rescales O.
// The roles' loops run side by side out of one instruction cache, and with 140 KB of code its misses set the pace.  So one
// warp walks the share of the work and tells the others the units (WideTask), waits and loads of queries are out of line, and
// what few items need (caps, hidden rows) is a rolled loop over tensor memory.
// 94 KB of code instead of 140: 32 tokens of 4 heads over 16 x 8 x 9728 rows of 128 channels 112 us instead of 119 (bytes 38.6; an
// fp8 cache without scales 130), 64 tokens over 2 x 8 x 131072 int8 rows 295 us (products 150).  No unit is full:
// tensor cores 27 %, DRAM 30 %, exponentials 28 % of their rates in the former; what is left are the chains of the softmax warps.
#pragma once
#include "lagkv_attend_quant_kernels.cuh"
#include "lagkv_attend_wide_kernel.cuh"
#include "lagkv_wide_walk.h"

namespace lagkv {

// int8 rows as the helpers widen them
struct WideInt8 {
    static __device__ __forceinline__ void expand(uint32_t w, uint32_t (&p)[2]) {  // 0x6400 | (c + 128) is 1152 + c in fp16
        const uint32_t u = w ^ 0x80808080u;
        asm("sub.f16x2 %0, %1, %2;" : "=r"(p[0]) : "r"(__byte_perm(u, 0x64646464u, 0x4140)), "r"(0x64806480u));
        asm("sub.f16x2 %0, %1, %2;" : "=r"(p[1]) : "r"(__byte_perm(u, 0x64646464u, 0x4342)), "r"(0x64806480u));
    }
};
template <int FORM>
struct WideCode : WideInt8 {};
template <>
struct WideCode<FORM_E4M3> : Elem<2> {};

constexpr int kWideTasks = 16;   // units that are announced: the loading warp is at most 8 ahead of the softmax

// A unit's part of a CTA's share; n = 0: there is none left.
struct WideTask {
    int b, u, tile0, n, first_cta, last_cta, len, tokens;
};

template <int D_, int FORM_, int MT_>
struct QuantWideGeo {
    static constexpr int D = D_, DT = 2, FORM = FORM_, MT = MT_;
    static constexpr bool NAN_ROWS = FORM_ == FORM_E4M3;
    static constexpr int ROWB = D, CPR = D / 16;
    static constexpr int PANELS = (D + 63) / 64, PANEL = kWideTile * 128, SLOT = PANELS * PANEL;
    static constexpr int EXCH = 32 * kWideTile * 4;  // MT = 1: 16 channels of each stream's O for the other
    static constexpr int QBYTES = MT == 2 ? 2 * SLOT : SLOT + EXCH;
    static constexpr int GROUPS = MT == 2 && D > 64 ? 2 : 3, HELP = 64;  // groups of helpers, their threads
    static constexpr int WARPS = 10 + 2 * GROUPS, NT = WARPS * 32;
    static constexpr int PASS = HELP / CPR & ~7, PASS_THREADS = PASS * CPR;
    static constexpr int SCALES = D == 64 ? 16 : 8;  // K tiles whose scales are kept: more than the rings hold
    static constexpr int MISC = 1024 + kWideTasks * int(sizeof(WideTask)) + SCALES * 16 * 4;
    static constexpr int RAW = kWideTile * ROWB, RS = GROUPS;  // (see WideGeo)
    static constexpr int NS_FIT = (232448 - 1024 - MISC - QBYTES - RS * RAW) / SLOT, NS = NS_FIT > 8 ? 8 : NS_FIT;
    static constexpr int SMEM = 1024 + QBYTES + NS * SLOT + RS * RAW + MISC;
    static constexpr int PSIZE = MT * kWideTile * (D + 2);
    static_assert(NS >= 4 && D <= 128 && D % 32 == 0, "does not fit");
};

__device__ __forceinline__ void tm_ld16(uint32_t (&r)[16], uint32_t a) {  // waited for
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(a)
        : "memory");
}

// mbar_wait_bounded() of which only the first look is inline: the instruction cache holds little more than the roles' loops.
static __device__ __noinline__ bool wide_wait_long(uint32_t bar, uint32_t parity) { return mbar_wait_bounded(bar, parity); }
__device__ __forceinline__ bool wide_wait(uint32_t bar, uint32_t parity) {
    return __all_sync(~0u, mbar_try_wait(bar, parity)) || wide_wait_long(bar, parity);
}

template <int D, int N>
__device__ __forceinline__ void quant_write_out(const QuantAttendParams& P, int b, int h, int m0, int tokens, int m, int d, const float (&o)[N],
                                                float ref, float sum) {
    if (P.half)
        attend_write<D, 1>(P, b, h, 0, m0, tokens, m, d, o, ref, sum);
    else
        attend_write<D, 0>(P, b, h, 0, m0, tokens, m, d, o, ref, sum);
}

// A task as the roles see it.
struct WideView {
    int b, h, m0, mrows, tile0, n, lim, base;  // query rows from m0 on; rows seen at all, first drafted row
    bool masked;
};
__device__ __forceinline__ WideView wide_view(const QuantAttendParams& P, const WideTask& k, int rows) {
    WideView v;
    v.b = k.b;
    v.h = k.u / P.mtiles;
    v.m0 = (k.u - v.h * P.mtiles) * rows;
    v.mrows = min(rows, P.T * P.G - v.m0);
    v.tile0 = k.tile0;
    v.n = k.n;
    v.lim = k.tokens == 0 ? 0 : k.len;
    v.base = k.len - k.tokens;
    v.masked = P.mask != nullptr || k.tokens > 1;
    return v;
}
// Loads of a task: V of step i is load load_of_v(i, n), K load_of_k(i).
template <int MT>
__device__ __forceinline__ bool load_is_v(int l, int n) { return MT == 2 ? (l & 1) != 0 : l == 2 * n - 1 || (l >= 2 && !(l & 1)); }
template <int MT>
__device__ __forceinline__ int load_step(int l, int n) {
    return MT == 2 ? l >> 1 : load_is_v<MT>(l, n) ? (l == 2 * n - 1 ? n - 1 : l / 2 - 1) : (l + 1) >> 1;
}

// The queries of a task into swizzled shared memory (`to`) and the exponents of the powers of two that their rows were scaled
// with (`factors`), by warp `warp` of `warps`: 8 or 16 lanes a row, several rows in flight.
template <class G>
__device__ __noinline__ void quant_load_queries(const QuantAttendParams& P, const WideTask* task, unsigned char* to, uint8_t* factors, int warp, int warps) {
    constexpr int CH = G::D / 8, LPR = CH > 8 ? 16 : 8, RPI = 32 / LPR, BATCH = 4;  // 16-byte pieces and lanes of a row, rows at a time, such steps in flight
    const WideView U = wide_view(P, *task, G::MT * kWideTile);
    const int lane = threadIdx.x & 31, ch = lane % LPR, sub = lane / LPR;
    const uint32_t by_g = ((1u << 20) + P.G - 1) / P.G;  // rows / G by a product: rows < 2^12, G <= 2^6
    const uint16_t* q0 = P.Q + (long long)U.b * P.q_sb + (long long)(U.h * P.G) * P.q_sh + ch * 8;
#pragma unroll 1
    for (int r0 = warp * RPI * BATCH; r0 < G::MT * kWideTile; r0 += warps * RPI * BATCH) {
        uint4 v[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int r = r0 + k * RPI + sub, row = U.m0 + r, t = int(row * by_g >> 20);
            v[k] = r < U.mrows && ch < CH ? __ldg(reinterpret_cast<const uint4*>(q0 + (long long)t * P.q_st + (long long)(row - t * P.G) * P.q_sh)) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int r = r0 + k * RPI + sub;
            float f = 1.f;
            if (!P.half) {
                float top = largest_of(v[k]);
#pragma unroll
                for (int o = LPR / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
                f = query_factor(top);
                uint32_t y[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = MmaHalf::pack(Elem<0>::lo(y[e]) * f, Elem<0>::hi(y[e]) * f);
                v[k] = make_uint4(y[0], y[1], y[2], y[3]);
            }
            if (ch == 0) factors[r] = uint8_t(__float_as_int(f) >> 23);
            if (ch < CH) *reinterpret_cast<uint4*>(to + (r >> 7) * G::SLOT + (ch >> 3) * G::PANEL + (r & 127) * 128 + (((ch & 7) ^ (r & 7)) << 4)) = v[k];
        }
    }
    fence_proxy_async();
    __syncwarp();
}

template <int D, int FORM, int MT>
__global__ void __launch_bounds__(QuantWideGeo<D, FORM, MT>::NT, 1)
lagkv_attend_quant_wide_kernel(const __grid_constant__ QuantAttendParams P, const __grid_constant__ CUtensorMap map_k,
                               const __grid_constant__ CUtensorMap map_v) {
    using G = QuantWideGeo<D, FORM, MT>;
    using C = WideCode<FORM>;
    extern __shared__ unsigned char raw[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, w = __shfl_sync(~0u, tid >> 5, 0);  // the same in all lanes, visibly
    const uint32_t sbase = (smem_u32(raw) + 1023u) & ~1023u;
    unsigned char* smem = raw + (sbase - smem_u32(raw));
    const uint32_t s_q = sbase, s_ring = sbase + G::QBYTES, s_raw = s_ring + G::NS * G::SLOT, s_misc = s_raw + G::RS * G::RAW;
    unsigned char* misc = smem + (s_misc - sbase);
    float* exch = reinterpret_cast<float*>(smem + G::SLOT);  // MT = 1
    // misc: barriers (tile ready, place free; landed, its place free; scores and probabilities of both streams' two places,
    // products of the streams; queries in place, their place free, the first ones in place; tasks told), the rows of each V tile
    // that are NaN, the missing 16-row groups of each load, exponents of the queries' factors (scheduling scratch before), tasks,
    // scales of K tiles' rows
    const uint32_t b_full = s_misc, b_empty = b_full + 8 * 8, b_land = b_empty + 8 * 8, b_raw_free = b_land + 4 * 8, b_s = b_raw_free + 4 * 8,
                   b_p = b_s + 4 * 8, b_o = b_p + 4 * 8, b_q = b_o + 2 * 8, b_q_free = b_q + 8, b_q_first = b_q_free + 8, b_task = b_q_first + 8;
    uint32_t* odd_rows = reinterpret_cast<uint32_t*>(misc + 432);                     // [8][4]
    volatile uint32_t* gone = reinterpret_cast<volatile uint32_t*>(misc + 560);       // [kWideRowFlags]
    uint32_t* tm_slot = reinterpret_cast<uint32_t*>(misc + 688);
    uint8_t* q_factors = misc + 704;                                                  // [MT * 128]
    long long* scan = reinterpret_cast<long long*>(misc + 704);                       // [16 + 2]
    WideTask* tasks = reinterpret_cast<WideTask*>(misc + 1024);                       // [kWideTasks]
    float* tile_scales = reinterpret_cast<float*>(misc + 1024 + kWideTasks * sizeof(WideTask));  // [SCALES][K, V][8]
    if (tid == 0) {
        for (int i = 0; i < G::NS; ++i) {
            mbar_init(b_full + 8 * i, 1);
            mbar_init(b_empty + 8 * i, 1);
        }
        for (int i = 0; i < G::RS; ++i) {
            mbar_init(b_land + 8 * i, 1);
            mbar_init(b_raw_free + 8 * i, 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(b_s + 8 * i, 1);
            mbar_init(b_p + 8 * i, 4);
        }
        for (int s = 0; s < 2; ++s) mbar_init(b_o + 8 * s, 1);
        mbar_init(b_q, 2 * G::GROUPS);
        mbar_init(b_q_free, 1);
        mbar_init(b_q_first, 8 + 2 * G::GROUPS);
        for (int i = 0; i < kWideTasks; ++i) mbar_init(b_task + 8 * i, 1);
        fence_mbar_init();
    }
    if (w == 8) {
        __syncwarp();
        tm_alloc(smem_u32(tm_slot));
        tm_fence_before();
    }
    const int upb = P.H * P.mtiles;
    AttendShare sh = attend_share<G::NT, kWideTile>(P, upb, scan);
    __syncthreads();
    tm_fence_after();
    const uint32_t tm = __shfl_sync(~0u, *reinterpret_cast<volatile uint32_t*>(tm_slot), 0);
    // tensor memory columns: scores (and probabilities over them) of stream s in place p, O of stream s
    auto at_s = [&](int s, int p) { return tm + (MT == 1 ? p * 128 + s * 64 : s * 128 + p * 64); };
    auto at_o = [&](int s) { return tm + 256 + s * D; };
    bool ok = true;
    // The task told in turn `k`, once it is; false: the last one is behind, or a wait was given up.  `agree`: see wide_go_on();
    // all threads of the barriers inside a task.
    auto next_task = [&](uint32_t k, WideView& U, auto&& agree) {
        auto told = [&]() {
            if (wide_wait(b_task + 8 * (k % kWideTasks), k / kWideTasks & 1)) return true;
            if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
            return false;
        };
        if (!wide_go_on(ok, told, agree)) return false;
        U = wide_view(P, tasks[k % kWideTasks], MT * kWideTile);
        return U.n > 0;
    };
    auto alone = [](bool mine) { return mine; };

    if (w == 9) {
        // ------------------------------------------------------------------ K and V tiles: a box per page, a lane each
        const int box_rows = P.block_table == nullptr ? kWideTile : min(kWideTile, 1 << P.page_shift);
        const uint32_t box_bytes = uint32_t(box_rows) * G::ROWB;
        uint32_t place = 0, lap = 0, c = 0;
        for (uint32_t task = 0; ok; ++task) {
            AttendSeq seq;
            AttendPart part;
            part.n = part.step = seq.tiles = 0;
            while (sh.pos < sh.end) {  // the next unit with rows
                seq = attend_seq<kWideTile>(P, sh.b, false);
                part = attend_part(P, sh, seq.tiles);
                if (part.n > 0) break;
                attend_advance(P, sh, part.step, seq.tiles, upb);
            }
            const int n = sh.pos < sh.end ? part.n : 0;
            if (lane == 0) {
                WideTask& k = tasks[task % kWideTasks];
                k.b = sh.b;
                k.u = part.u;
                k.tile0 = part.tile0;
                k.n = n;
                k.first_cta = int(part.c0);
                k.last_cta = int(part.c1);
                k.len = seq.len;
                k.tokens = seq.tokens;
                mbar_arrive(b_task + 8 * (task % kWideTasks));
            }
            if (n == 0) break;
            const int h = part.u / P.mtiles, lim = seq.tokens == 0 ? 0 : seq.len;
            for (int l = 0; l < 2 * n && ok; ++l, ++c) {
                const bool is_v = load_is_v<MT>(l, n);
                const int row = (part.tile0 + load_step<MT>(l, n)) * kWideTile + lane * box_rows;
                bool there = lane < kWideTile / box_rows && row < lim;
                const bool wanted = there;
                int c1 = row, c3 = sh.b;
                if (there && P.block_table != nullptr) {
                    c3 = __ldg(P.block_table + (long long)sh.b * P.max_blocks + (row >> P.page_shift));
                    c1 = row & ((1 << P.page_shift) - 1);
                    if (c3 < 0 || c3 >= P.num_pages) {
                        there = false;
                        record_status(P.status, ST_EINVAL, sh.b);
                    }
                }
                const int boxes = __popc(__ballot_sync(~0u, there));
                uint32_t flags = 0;  // a bit per group of 16 rows whose page is not in the pool
                for (unsigned m = __ballot_sync(~0u, wanted && !there); m; m &= m - 1)
                    flags |= ((1u << box_rows / 16) - 1) << (__ffs(int(m)) - 1) * box_rows / 16;
                if (lap > 0 && !wide_wait(b_raw_free + 8 * place, (lap + 1) & 1)) {
                    if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
                    ok = false;
                    break;
                }
                if (lane == 0) {
                    gone[c % kWideRowFlags] = flags;
                    mbar_arrive_expect_tx(b_land + 8 * place, boxes * box_bytes);
                }
                __syncwarp();
                if (there)
                    asm volatile(
                        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
                            s_raw + place * G::RAW + lane * box_bytes),
                        "l"(is_v ? &map_v : &map_k), "r"(0), "r"(c1), "r"(h), "r"(c3), "r"(b_land + 8 * place)
                        : "memory");
                __syncwarp();
                if (++place == uint32_t(G::RS)) place = 0, ++lap;
            }
            attend_advance(P, sh, part.step, seq.tiles, upb);
        }
    } else if (w > 9) {
        // ------------------------------------------------------------------ help: queries, and tiles widened, a group every GROUPS-th
        const int group = (w - 10) / 2, ptid = tid - 10 * 32 - group * G::HELP;
        // after a wait that ran out this warp goes on to the end of its task without waiting, so that it comes to every barrier of
        // its group: how many a tile has follows from the task alone.  Then the group leaves together.
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (ok && !wide_wait(bar, parity)) {
                if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
                ok = false;
            }
        };
        auto meet = [&]() { named_bar_sync(2 + group, G::HELP); };
        auto agree = [&](bool mine) { return !named_bar_or(2 + group, G::HELP, !mine); };
        uint32_t lap = 0, slot_lap = 0, c = 0;  // how often this group's place and the load's slot have been through; loads before
        int turn = 0, slot = 0;
        WideView U;
        for (uint32_t task = 0; next_task(task, U, agree); ++task) {
            // the task's queries, once the products with those before are done
            if (task > 0) wait(b_q_free, (task - 1) & 1);
            quant_load_queries<G>(P, tasks + task % kWideTasks, smem, q_factors, task > 0 ? w - 10 : w - 2, 2 * G::GROUPS + (task > 0 ? 0 : 8));
            if (lane == 0 && ok) mbar_arrive(task > 0 ? b_q : b_q_first);
#pragma unroll 1
            for (int l = 0; l < 2 * U.n; ++l, ++c) {
                const bool mine = turn == group;
                const int at_slot = slot;
                const uint32_t at_lap = lap, at_slot_lap = slot_lap;
                if (++turn == G::GROUPS) turn = 0, ++lap;
                if (++slot == G::NS) slot = 0, ++slot_lap;
                if (!mine) continue;
                const bool is_v = load_is_v<MT>(l, U.n);
                const int row0 = (U.tile0 + load_step<MT>(l, U.n)) * kWideTile;
                if (!is_v && ptid < 16) {  // with the K tile come the scales of its rows, V's too
                    const int row = row0 + 16 * (ptid & 7);
                    const long long s = ((long long)U.b * P.H + U.h) * P.blocks + (row >> P.block_shift);
                    tile_scales[((c + 1) / 2 % G::SCALES) * 16 + ptid] = row < U.lim ? __ldg((ptid < 8 ? P.K_scale : P.V_scale) + s) : 0.f;
                }
                wait(b_land + 8 * group, at_lap & 1);
                const uint32_t groups = is_v ? gone[c % kWideRowFlags] : 0u;
                const bool careful = G::NAN_ROWS && is_v && U.masked && row0 + kWideTile > U.base;
                const bool mend = is_v && (P.block_table != nullptr || careful || row0 + kWideTile > U.lim);
                unsigned char* tile = smem + (s_ring - sbase) + at_slot * G::SLOT;
                if (at_slot_lap > 0) wait(b_empty + 8 * at_slot, (at_slot_lap + 1) & 1);
                const unsigned char* from = smem + (s_raw - sbase) + group * G::RAW;
                if (careful) {  // drafted rows that are NaN; rows of `groups` have no page, their place holds what an older tile left there
                    if (ptid < 4) odd_rows[at_slot * 4 + ptid] = 0u;
                    meet();
                    const int first = max(0, U.base - row0) * G::CPR, last = min(kWideTile, U.lim - row0) * G::CPR;
#pragma unroll 4
                    for (int id = first + ptid; id < last; id += G::HELP) {
                        const uint4 v = *reinterpret_cast<const uint4*>(from + id * 16);
                        const uint32_t nan = Code<FORM>::nan_bytes(v.x) | Code<FORM>::nan_bytes(v.y) | Code<FORM>::nan_bytes(v.z) | Code<FORM>::nan_bytes(v.w);
                        if (nan && !(groups >> (id / G::CPR >> 4) & 1)) atomicOr(&odd_rows[at_slot * 4 + id / G::CPR / 32], 1u << (id / G::CPR & 31));
                    }
                    meet();
                }
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
                        C::expand(x.x, a);
                        C::expand(x.y, b);
                        C::expand(x.z, e);
                        C::expand(x.w, f);
                        *reinterpret_cast<uint4*>(to + c0 + i * G::PASS * 128) = make_uint4(a[0], a[1], b[0], b[1]);
                        *reinterpret_cast<uint4*>(to + c1 + i * G::PASS * 128) = make_uint4(e[0], e[1], f[0], f[1]);
                    }
                }
                if (mend) {  // rows behind the last one, without a page, or noted become zeros, so that 0 * NaN never happens
                    meet();
                    const uint32_t* odd = odd_rows + at_slot * 4;
                    const int begin = groups ? 0 : max(0, (careful && (odd[0] | odd[1] | odd[2] | odd[3]) ? min(U.base, U.lim) : U.lim) - row0);
                    for (int id = begin * (D / 8) + ptid; id < kWideTile * (D / 8); id += G::HELP) {
                        const int rr = id / (D / 8), cc = id % (D / 8);
                        if (row0 + rr >= U.lim || (groups >> (rr >> 4) & 1) || (careful && (odd[rr >> 5] >> (rr & 31) & 1)))
                            *reinterpret_cast<uint4*>(tile + (cc >> 3) * G::PANEL + rr * 128 + (((cc & 7) ^ (rr & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                    }
                }
                fence_proxy_async();
                meet();
                if (ptid == 0 && ok) {
                    mbar_arrive(b_full + 8 * at_slot);
                    mbar_arrive(b_raw_free + 8 * group);
                }
            }
        }
    } else if (w == 8) {
        // ------------------------------------------------------------------ the products
        constexpr uint32_t id_qk = mma_idesc(false, false, MT == 1 ? 128 : 64), id_pv = mma_idesc(false, true, D);
        const uint32_t lead = elect_one();
        uint32_t slot = G::NS - 1, phase = 1;  // the load taken last (loads are taken in their order)
        uint32_t np = 0;                       // parities of the probabilities (a bit per stream and place)
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (ok && !wide_wait(bar, parity)) {
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
        // scores of stream s (MT = 1: of both) against rows 64 half .. of the K tile in `k_slot`
        auto scores = [&](int s, int p, uint32_t k_slot, int half) {
            // addresses count in 16 bytes in the low word and never carry out of it
            const uint32_t q = smem_desc_lo(s_q + (MT == 2 ? s * G::SLOT : 0), 16), kd = smem_desc_lo(s_ring + k_slot * G::SLOT, 16) + half * (64 * 128 >> 4);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const uint32_t o = ((ks >> 2) * G::PANEL + (ks & 3) * 32) >> 4;
                mma_ss(lead, at_s(s, p), q + o, kd + o, id_qk, ks != 0);
            }
            tm_commit(lead, b_s + 8 * (2 * s + p));
            if (MT == 1) tm_commit(lead, b_s + 8 * (2 + p));
        };
        // O += P V of the item of stream s in place p: rows 64 half .. of the V tile
        auto outputs = [&](int s, int p, uint32_t v_slot, int half) {
            const int bit = 2 * s + p;
            if (!wait(b_p + 8 * bit, np >> bit & 1)) return;
            np ^= 1u << bit;
            tm_fence_after();
            const uint32_t v = smem_desc_lo(s_ring + v_slot * G::SLOT, G::PANEL) + half * (64 * 128 >> 4);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) mma_ts(lead, at_o(s), at_s(s, p) + ks * 8, v + ks * (2048 >> 4), id_pv);
            tm_commit(lead, b_o + 8 * s);
        };
        WideView U;
        for (uint32_t task = 0; next_task(task, U, alone); ++task) {
            const int n = __shfl_sync(~0u, U.n, 0);
            if (!wait(task > 0 ? b_q : b_q_first, task > 0 ? (task - 1) & 1 : 0)) break;
            if constexpr (MT == 1) {
                // step i: products with V of tile i, and the scores of tile i + 2, whose place they free
#pragma unroll 1
                for (int i = -2; i < n && ok; ++i) {
                    if (i >= 0) {
                        if (!next_load()) break;
                        const uint32_t v_slot = slot;
#pragma unroll 1
                        for (int s = 0; s < 2 && ok; ++s) outputs(s, i & 1, v_slot, s);
                        if (!ok) break;
                        tm_commit(lead, b_empty + 8 * v_slot);
                    }
                    if (i + 2 < n) {
                        // K of the first two tiles come before V of the first, then K of tile i + 2 before V of tile i + 1
                        if (!next_load()) break;
                        scores(0, i & 1, slot, 0);
                        tm_commit(lead, b_empty + 8 * slot);
                    }
                    // behind the unit's last scores, and behind probabilities of both streams, which have read the rows' factors by then
                    if (i == max(n - 3, 0)) tm_commit(lead, b_q_free);
                }
            } else {
                // step j: products with half j of the V tiles, and the scores of half j + 2
                uint32_t v_slot = 0, k_slot = 0;
                if (!next_load()) break;
                k_slot = slot;
#pragma unroll 1
                for (int j = -2; j < 2 * n && ok; ++j) {
                    const bool has_v = j >= 0, has_k = j + 2 < 2 * n;
                    if (has_v && !(j & 1)) {
                        if (!next_load()) break;
                        v_slot = slot;
                        if (has_k) {
                            if (!next_load()) break;
                            k_slot = slot;
                        }
                    }
#pragma unroll 1
                    for (int s = 0; s < 2 && ok; ++s) {
                        if (has_v) outputs(s, j & 1, v_slot, j & 1);
                        if (ok && has_k) scores(s, j & 1, k_slot, j & 1);
                    }
                    if (!ok) break;
                    if (has_v && (j & 1)) tm_commit(lead, b_empty + 8 * v_slot);
                    if (has_k && (j & 1)) tm_commit(lead, b_empty + 8 * k_slot);
                    if (j == max(2 * n - 3, 0)) tm_commit(lead, b_q_free);  // (see above)
                }
            }
        }
    } else {
        // ------------------------------------------------------------------ softmax of a stream
        const int s = w >> 2, m = tid & 127;
        const uint32_t lanes = uint32_t(w & 3) << 21;  // tensor memory lanes 32 (w % 4) ..
        const uint32_t t_o = at_o(s) + lanes;
        uint32_t ns = 0, items = 0, c0 = 0;  // parities of the scores (a bit per place); items and loads of the units before
        auto wait = [&](uint32_t bar, uint32_t parity) {
            // after a wait that ran out the barriers of this task go on, everything else stops; then all these warps leave together
            if (ok && !wide_wait(bar, parity)) {
                if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
                ok = false;
            }
            tm_fence_after();
        };
        // up to 128 query rows: the streams meet to join their results; else no warp waits for another at a barrier
        auto agree = [&](bool mine) { return MT == 1 ? !named_bar_or(1, 256, !mine) : mine; };
        WideView U;
        for (uint32_t task = 0; next_task(task, U, agree); ++task) {
            const WideTask& told = tasks[task % kWideTasks];
            if (task == 0) {  // the first queries
                quant_load_queries<G>(P, &told, smem, q_factors, w, 8 + 2 * G::GROUPS);
                if (lane == 0) mbar_arrive(b_q_first);
            }
            const int tokens = told.tokens;
            const int mine = MT == 2 ? 2 * U.n : U.n;          // items of this stream
            const int mu = (MT == 2 ? s * kWideTile : 0) + m;  // this thread's query row in the unit
            const int row = U.m0 + mu, t = row / P.G;
            const bool there = mu < U.mrows;
            unsigned long long bits = 0;
            if (there && U.masked && t < tokens)
                bits = P.mask ? P.mask[(long long)U.b * P.T + t] : (t == 63 ? ~0ull : (2ull << t) - 1);
            __syncwarp();  // the instructions on tensor memory need warps that are together
            {  // O starts at zero, every product adds to it
                uint32_t z[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) z[k] = 0u;
#pragma unroll
                for (int d = 0; d < D; d += 32) tm_st32(t_o + d, z);
                tm_wait_st();
            }
            float ref = -INFINITY, sum = 0.f, scl = 0.f;
            int ve = -126;  // O counts in units of 2^ve
#pragma unroll 1
            for (int k = 0; k < mine; ++k) {
                const int i = MT == 2 ? k >> 1 : k, half = MT == 2 ? k & 1 : s, p = k & 1;
                const uint32_t t_s = at_s(s, p) + lanes;
                const int r0 = (U.tile0 + i) * kWideTile + 64 * half;
                wait(b_s + 8 * (2 * s + p), ns >> p & 1);
                ns ^= 1u << p;
                if (k == 0) scl = P.scale_log2 / __int_as_float(int(q_factors[mu]) << 23);  // written before the scores were
                const uint32_t load = c0 + load_of_k<MT>(i);
                const float* scales = tile_scales + ((load + 1) / 2 % G::SCALES) * 16 + 4 * half;
                const bool draft = U.masked && r0 + 64 > U.base;
                const uint32_t missing = gone[load % kWideRowFlags] >> 4 * half & 15u;  // 16-row groups without a page
                const bool hidden = draft || missing || r0 + 64 > U.lim;
                // which of 32 rows from r on this query row sees
                auto seen32 = [&](int r) -> uint32_t {
                    uint32_t see = r >= U.lim ? 0u : U.lim - r >= 32 ? ~0u : (1u << (U.lim - r)) - 1;
                    if (missing >> ((r - r0) >> 4) & 1) see &= 0xffff0000u;
                    if (missing >> ((r - r0) >> 4) & 2) see &= 0x0000ffffu;
                    if (draft && r + 32 > U.base) {
                        const int j = r - U.base;  // drafted rows j ..
                        see &= j >= 64 ? 0u : j >= 0 ? uint32_t(bits >> j) : (j > -32 ? uint32_t(bits << -j) | ((1u << -j) - 1) : ~0u);
                    }
                    return see;
                };
                if (hidden || P.cap_inv != 0.f) {  // in place, out of the way of what every item runs (see the end of the file's head)
#pragma unroll 1
                    for (int q = 0; q < 4; ++q) {
                        uint32_t x[16];
                        tm_ld16(x, t_s + 16 * q);
                        if (P.cap_inv != 0.f) {
                            const float fx = fmaxf(scl * scales[q], 0x1p-126f) * P.cap_inv;
#pragma unroll
                            for (int e = 0; e < 16; ++e) x[e] = __float_as_uint(P.cap_log2 * quant_tanh(__uint_as_float(x[e]) * fx));
                        }
                        const uint32_t see = seen32(r0 + 32 * (q >> 1)) >> 16 * (q & 1);
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (!(see >> e & 1)) x[e] = 0xff800000u;
                        __syncwarp();
                        tm_st16(t_s + 16 * q, x);
                    }
                    tm_wait_st();
                }
                uint32_t a[32], b[32];
                tm_ld32(a, t_s);
                tm_ld32(b, t_s + 32);
                // factors of the logits of 16 rows each: never 0, which would make NaN of the -infinity of hidden rows
                float fk[4], vmax = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    fk[e] = P.cap_inv != 0.f ? 1.f : fmaxf(scl * scales[e], 0x1p-126f);
                    vmax = fmaxf(vmax, scales[8 + e]);
                }
                tm_wait_ld(a);
                tm_wait_ld(b);
                float top = -INFINITY;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x = -INFINITY, y = -INFINITY;
#pragma unroll
                    for (int e = 16 * h; e < 16 * h + 16; e += 2) {
                        x = fmaxf(x, fmaxf(__uint_as_float(a[e]), __uint_as_float(a[e + 1])));
                        y = fmaxf(y, fmaxf(__uint_as_float(b[e]), __uint_as_float(b[e + 1])));
                    }
                    top = fmaxf(top, fmaxf(x * fk[h], y * fk[2 + h]));
                }
                // The reference moves only when a probability would pass 2^6 of what it was set for, 2^ve when a V scale passes
                // its double: 2^8 * 2^6 * 2 fits fp16.
                top -= MmaHalf::kRefShift;
                const bool first = ref == -INFINITY, grew = top > ref + 6.f || (first && top > -INFINITY);
                const int to = min(((__float_as_int(vmax) >> 23) & 255) - 126, 126);  // vmax < 2^to
                const bool wider = to > ve + 1;  // the same for all rows
                bool waited = k == 0;
                auto before = [&]() {  // the product of the item before has to be over
                    if (!waited) wait(b_o + 8 * s, (items + k - 1) & 1);
                    waited = true;
                };
                if (__any_sync(~0u, grew && !first) || (wider && k > 0)) {
                    before();
                    float g = grew && !first ? ex2(ref - top) : 1.f;
                    sum *= g;
                    if (wider) g *= ve - to < -126 ? 0.f : pow2_of(ve - to);
#pragma unroll 1
                    for (int d = 0; d < D; d += 16) {
                        uint32_t o[16];
                        tm_ld16(o, t_o + d);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * g);
                        tm_st16(t_o + d, o);
                    }
                    tm_wait_st();
                }
                if (wider) ve = to;
                if (grew) ref = top;
                const float at = ref == -INFINITY ? 0.f : ref, unit = pow2_of(-ve);
                if (G::NAN_ROWS && draft) {
                    // drafted rows with NaN went into the tile as zeros: those who see them get NaN
                    const uint32_t l = c0 + load_of_v<MT>(i, U.n);
                    wait(b_full + 8 * (l % G::NS), (l / G::NS) & 1);
                    const uint32_t* noted = odd_rows + l % G::NS * 4 + 2 * half;
#pragma unroll 1
                    for (int x = 0; x < 2; ++x) {
#pragma unroll 1
                        for (uint32_t odd = ok ? noted[x] : 0u; odd; odd &= odd - 1) {
                            before();
                            const int e = __ffs(int(odd)) - 1, r = r0 + 32 * x + e;
                            const bool see = seen32(r0 + 32 * x) >> e & 1;
                            const long long off = attend_offset(P, U.b, U.h, r & ~15);
                            if (off < 0) continue;  // no page: never noted
                            const float z = __uint_as_float(tm_read1(t_s + 32 * x + e));
                            const float prob = see ? ex2(z * fk[2 * x + e / 16] - at) * scales[8 + 2 * x + e / 16] * unit : 0.f;
                            const uint8_t* v = P.V + off + (long long)(r & 15) * P.ss;
#pragma unroll 1
                            for (int d = 0; d < D; d += 16) {
                                uint32_t o[16];
                                tm_ld16(o, t_o + d);
#pragma unroll
                                for (int c = 0; c < 16; ++c) {
                                    uint32_t pr[2];
                                    C::expand(__ldg(v + d + c), pr);
                                    if (see) o[c] = __float_as_uint(__uint_as_float(o[c]) + prob * Elem<1>::lo(pr[0]));
                                }
                                __syncwarp();
                                tm_st16(t_o + d, o);
                                tm_wait_st();
                            }
                        }
                    }
                }
                // probabilities: their sums in fp32, then times V's scale, in 16 bits, over the scores
                {
                    const f32x2 at2 = pack2(-at, -at);
                    f32x2 part[2] = {0ull, 0ull};
                    uint32_t pr[32];
                    auto step = [&](const uint32_t (&x)[32], int e, int h, uint32_t& to16) {
                        float p0, p1;
                        unpack2(fma2(pack2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), pack2(fk[h], fk[h]), at2), p0, p1);
                        const f32x2 pp = pack2(ex2(p0), ex2(p1));
                        part[e / 2 & 1] = add2(part[e / 2 & 1], pp);
                        const float v = scales[8 + h] * unit;
                        unpack2(mul2(pp, pack2(v, v)), p0, p1);
                        to16 = MmaHalf::pack(p0, p1);
                    };
#pragma unroll
                    for (int e = 0; e < 32; e += 2) step(a, e, e / 16, pr[e / 2]);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) step(b, e, 2 + e / 16, pr[16 + e / 2]);
                    tm_st32(t_s, pr);
                    float s0, s1;
                    unpack2(add2(part[0], part[1]), s0, s1);
                    sum += s0 + s1;
                }
                before();
                tm_wait_st();
                tm_fence_before();
                __syncwarp();
                if (lane == 0 && ok) mbar_arrive(b_p + 8 * (2 * s + p));
            }
            if (mine > 0) wait(b_o + 8 * s, (items + mine - 1) & 1);
            items += mine;

            // ---- the unit's result
            const int first_cta = told.first_cta, last_cta = told.last_cta;
            const bool shared = first_cta != last_cta, writes = there && ok;
            float* part = P.partials + (2ll * blockIdx.x + (first_cta == int(blockIdx.x) ? 1 : 0)) * G::PSIZE + (MT == 2 ? s * kWideTile * (D + 2) : 0) + m;
            float mref = ref, msum = sum, f_own = 1.f;
            if (MT == 1) {  // both streams' references and sums; each finishes every other group of 16 channels
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
            f_own *= pow2_of(ve);
            // not shared: out and lse, as attend_write() has them
            const long long at_row = (((long long)U.b * P.T + t) * P.H + U.h) * P.G + (row - t * P.G);
            const bool live = t < tokens && msum != 0.f;  // NaN sums stay: they compare unequal to 0
            const float inv = live ? P.v_scale / msum : 0.f;
            if (writes && (MT == 2 || s == 0)) {
                if (shared)
                    __stcg(reinterpret_cast<float2*>(part - m + kWideTile * D + 2 * m), make_float2(mref, msum));
                else if (P.lse)
                    P.lse[at_row] = live ? 0.69314718055994531f * (mref + log2f(msum)) : -INFINITY;
            }
#pragma unroll 1
            for (int d0 = 0; d0 < D; d0 += MT == 1 ? 32 : 16) {
                uint32_t a[16];
                __syncwarp();
                if (MT == 1) {  // hands over its part of the other's channels
                    tm_ld16(a, t_o + d0 + 16 * (s ^ 1));
#pragma unroll
                    for (int e = 0; e < 16; ++e) exch[(s * 16 + e) * kWideTile + m] = __uint_as_float(a[e]) * f_own;
                    named_bar_sync(1, 256);
                }
                const int d = d0 + (MT == 1 ? 16 * s : 0);
                tm_ld16(a, t_o + d);
                float o[16];
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    o[e] = MT == 1 ? __uint_as_float(a[e]) * f_own + exch[((s ^ 1) * 16 + e) * kWideTile + m] : __uint_as_float(a[e]) * f_own;
                if (writes && shared) {  // channel by channel: a warp writes 32 rows side by side
#pragma unroll
                    for (int e = 0; e < 16; ++e) __stcg(part + (d + e) * kWideTile, o[e]);
                } else if (writes) {
                    uint32_t v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = o[2 * e] * inv, y = o[2 * e + 1] * inv;
                        v[e] = !live ? 0u : P.half ? MmaHalf::pack(x, y) : Mma<0>::pack(x, y);
                    }
                    uint4* to = reinterpret_cast<uint4*>(P.out + at_row * D + d);
                    to[0] = make_uint4(v[0], v[1], v[2], v[3]);
                    to[1] = make_uint4(v[4], v[5], v[6], v[7]);
                }
                __syncwarp();
                if (MT == 1) named_bar_sync(1, 256);
            }
            // who shares the unit, for the kernel that joins the partials: said once, by the CTA that starts it
            if (tid == 0 && first_cta == int(blockIdx.x))
                P.shared[(long long)U.b * upb + told.u] = ok ? make_int2(first_cta, last_cta) : make_int2(0, 0);
            c0 += 2 * U.n;
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

template <int D, int FORM, int MT>
__global__ void __launch_bounds__(kJoinThreads)
lagkv_attend_quant_join_kernel(const __grid_constant__ QuantAttendParams P) {
    attend_join<D, MT>(P, [&](int b, int h, int m0, int tokens, int m, int d, const auto& o, float top, float total) {
        quant_write_out<D>(P, b, h, m0, tokens, m, d, o, top, total);
    });
}

}  // namespace lagkv
