// Attention over the cache for many query rows (wide trees) -- 5th-generation tensor cores.
//
// The same mathematics and the same shares of the work as lagkv_attend_kernel.  With 33 or more query rows
// per KV head the products of a 128-row tile outgrow mma.sync (that kernel reached 150 TFLOP/s); here they
// run as tcgen05.mma with M = 128 query rows, accumulators and probabilities in tensor memory:
//     S[128 x 128] = Q K^T (both from shared memory),   O[128 x D] += P V (P from tensor memory).
// Two streams keep the tensor cores busy while the other one's softmax runs: with up to 128 query rows the
// streams take every other tile of rows and are joined at the end, with up to 256 each has its own 128
// query rows and both read the same tiles.
// Warps: 0-3 and 4-7 the softmax of stream 0 and 1 (a thread owns a query row), 8-11 fetch K and V tiles
// into swizzled shared memory (cp.async: rows are found page by page and rows behind the last one are
// zero-filled, which a tensor map cannot do; fp8 rows are widened to fp16 on the way), 12 issues.
// Bound: at 128 rows and 16-bit caches by HBM, at 256 by the 16384 exponentials per tile and stream (16 a
// cycle and SM: as long as the products themselves).
#pragma once
#include "lagkv_attend_kernels.cuh"

namespace lagkv {

constexpr int kWideTile = 128;        // rows of K and V per step
constexpr int kWideThreads = 13 * 32;
constexpr int kWideLag = 2;           // tiles whose copies are in flight behind the one being issued

template <int D_, int DT_, int MT_>
struct WideGeo {
    static constexpr int D = D_, DT = DT_, MT = MT_;  // MT = 1: streams split the rows, 2: the query rows
    static constexpr int EB = Elem<DT_>::EB;
    static constexpr int ROWB = D * EB, CPR = ROWB / 16;
    static constexpr int PANELS = (D + 63) / 64;       // 64 channels of 16 bits: 128-byte rows, swizzled
    static constexpr int PANEL = kWideTile * 128;
    static constexpr int SLOT = PANELS * PANEL;
    static constexpr int EXCH = 64 * kWideTile * 4;    // MT = 1: 64 channels of one stream's O for the other
    static constexpr int QBYTES = MT == 2 ? 2 * SLOT : SLOT + EXCH;
    static constexpr int MISC = 1024;
    static constexpr int NS_FIT = (232448 - 1024 - MISC - QBYTES) / SLOT;
    static constexpr int NS = NS_FIT > 8 ? 8 : NS_FIT; // tiles of K or V in the ring
    static constexpr int SMEM = 1024 + QBYTES + NS * SLOT + MISC;
    static constexpr int PSIZE = MT * kWideTile * (D + 2);
    static_assert(NS >= 5, "the order of the ring needs five tiles");
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
__device__ __forceinline__ void tm_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(1)
        : "memory");
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

// Shared memory operand: 128-byte rows in groups of eight (1024 bytes), swizzled by 128 bytes.  `lead`: bytes
// between panels of 64 channels (read when the panels run along the operand's outer dimension, as in V).
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead) {
    return uint64_t((addr & 0x3ffff) >> 4) | uint64_t(lead >> 4) << 16 | uint64_t(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
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
    int lim, base;                  // rows seen at all, first drafted row
    bool masked;
};
template <class G>
__device__ __forceinline__ WideUnit wide_unit(const AttendParams& P, const AttendShare& sh) {
    WideUnit w;
    w.seq = attend_seq<kWideTile>(P, sh.b, false);
    w.u = int((sh.pos - sh.first) / w.seq.tiles);
    w.tile0 = int((sh.pos - sh.first) % w.seq.tiles);
    w.n = int(min((long long)(w.seq.tiles - w.tile0), sh.end - sh.pos));
    w.h = w.u / P.mtiles % P.H;
    w.m0 = w.u % P.mtiles * (G::MT * kWideTile);
    w.mrows = min(G::MT * kWideTile, P.T * P.G - w.m0);
    w.lim = w.seq.tokens == 0 ? 0 : w.seq.len;
    w.base = w.seq.len - w.seq.tokens;
    w.masked = P.mask != nullptr || w.seq.tokens > 1;
    return w;
}
__device__ __forceinline__ void wide_next(AttendShare& sh, const WideUnit& w, int units_per_seq) {
    sh.pos += w.n;
    if (sh.pos == sh.first + (long long)units_per_seq * w.seq.tiles) {
        sh.first = sh.pos;
        ++sh.b;
    }
}

template <int D, int DT, int MT>
__global__ void __launch_bounds__(kWideThreads, 1)
lagkv_attend_wide_kernel(const __grid_constant__ AttendParams P) {
    using G = WideGeo<D, DT, MT>;
    using X = Mma<DT>;
    extern __shared__ unsigned char raw[];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const uint32_t sbase = (smem_u32(raw) + 1023u) & ~1023u;
    unsigned char* smem = raw + (sbase - smem_u32(raw));
    const uint32_t s_q = sbase, s_ring = sbase + G::QBYTES, s_misc = s_ring + G::NS * G::SLOT;
    unsigned char* misc = smem + G::QBYTES + G::NS * G::SLOT;
    float* exch = reinterpret_cast<float*>(smem + G::SLOT);  // MT = 1
    // misc: barriers, the rows of each V tile that are not finite, scheduling scratch
    const uint32_t b_full = s_misc, b_empty = s_misc + 8 * 8, b_s = s_misc + 16 * 8, b_p = b_s + 16, b_o = b_p + 16, b_q = b_o + 16;
    uint32_t* odd_rows = reinterpret_cast<uint32_t*>(misc + 256);  // [8][4]
    long long* scan = reinterpret_cast<long long*>(misc + 512);    // [13 + 2]
    uint32_t* tm_slot = reinterpret_cast<uint32_t*>(misc + 640);
    int* slast = reinterpret_cast<int*>(misc + 644);

    if (tid == 0) {
        for (int i = 0; i < G::NS; ++i) {
            mbar_init(b_full + 8 * i, 4);
            mbar_init(b_empty + 8 * i, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(b_s + 8 * s, 1);
            mbar_init(b_p + 8 * s, 4);
            mbar_init(b_o + 8 * s, 1);
        }
        mbar_init(b_q, 8);
        fence_mbar_init();
    }
    if (w == 12) {
        __syncwarp();
        tm_alloc(smem_u32(tm_slot));
        tm_fence_before();
    }
    const int upb = P.H * P.mtiles;
    AttendShare sh = attend_share<kWideThreads, kWideTile>(P, upb, scan);
    __syncthreads();
    tm_fence_after();
    const uint32_t tm = *reinterpret_cast<volatile uint32_t*>(tm_slot);
    // tensor memory columns: S (and P over it) of stream 0, 1 at 0, 128; O at 256, 256 + D
    constexpr int kO = 256;
    bool ok = true;

    if (w >= 8 && w < 12) {
        // ------------------------------------------------------------------ K and V tiles
        const int ptid = tid - 256;
        uint32_t c = 0;  // loads so far
        auto signal = [&](uint32_t k) {
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(b_full + 8 * (k % G::NS));
        };
        for (; ok && sh.pos < sh.end;) {
            const WideUnit U = wide_unit<G>(P, sh);
            for (int l = 0; ok && l < 2 * U.n; ++l, ++c) {
                // which tile is load l
                int i;
                bool is_v;
                if (MT == 2) {
                    i = l >> 1;
                    is_v = l & 1;
                } else {
                    is_v = l == 2 * U.n - 1 || (l >= 2 && !(l & 1));
                    i = is_v ? (l == 2 * U.n - 1 ? U.n - 1 : l / 2 - 1) : (l + 1) >> 1;
                }
                const int slot = int(c % G::NS), r0 = (U.tile0 + i) * kWideTile;
                if (c >= uint32_t(G::NS) && !mbar_wait_bounded(b_empty + 8 * slot, (c / G::NS + 1) & 1)) {
                    if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
                    ok = false;
                    break;
                }
                const uint8_t* T = is_v ? P.V : P.K;
                // lanes 0-7: offsets of the tile's eight groups of 16 rows
                long long off = -1;
                if (lane < 8 && r0 + 16 * lane < U.lim) off = attend_offset(P, sh.b, U.h, r0 + 16 * lane);
                const uint32_t dst = s_ring + slot * G::SLOT;
                const bool careful = is_v && U.masked && r0 + kWideTile > U.base;
                if (careful) {
                    if (ptid < 4) odd_rows[slot * 4 + ptid] = 0u;
                    asm volatile("bar.sync 2, 128;" ::: "memory");
                }
                if constexpr (DT != 2) {
                    if (!careful) {
#pragma unroll
                        for (int j = 0; j < kWideTile * G::CPR / 128; ++j) {
                            const int id = j * 128 + ptid, r = id / G::CPR, ch = id % G::CPR;
                            const long long o = __shfl_sync(~0u, off, r >> 4);
                            const bool there = o >= 0 && r0 + r < U.lim;
                            cp_async16(dst + (ch >> 3) * G::PANEL + r * 128 + (((ch & 7) ^ (r & 7)) << 4),
                                       T + (there ? o + (long long)(r & 15) * P.ss + ch * 16 : 0), there);
                        }
                    }
                }
                if (DT == 2 || careful) {
                    // through registers: fp8 rows widen to fp16; of a drafted V tile the rows that are not
                    // finite are noted and enter as zeros
                    constexpr int N = kWideTile * G::CPR / 128;
                    uint4 v[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const int id = j * 128 + ptid, r = id / G::CPR, ch = id % G::CPR;
                        const long long o = __shfl_sync(~0u, off, r >> 4);
                        const bool there = o >= 0 && r0 + r < U.lim;
                        v[j] = there ? __ldg(reinterpret_cast<const uint4*>(T + o + (long long)(r & 15) * P.ss + ch * 16)) : make_uint4(0u, 0u, 0u, 0u);
                    }
                    if (careful) {
#pragma unroll
                        for (int j = 0; j < N; ++j) {
                            const int r = (j * 128 + ptid) / G::CPR;
                            const uint32_t x[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
                            bool odd = false;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                if (DT == 0) odd |= (x[k] & 0x7f80u) == 0x7f80u || (x[k] & 0x7f800000u) == 0x7f800000u;
                                if (DT == 1) odd |= (x[k] & 0x7c00u) == 0x7c00u || (x[k] & 0x7c000000u) == 0x7c000000u;
                                if (DT == 2)
                                    for (int e = 0; e < 4; ++e) odd |= ((x[k] >> (8 * e)) & 0x7f) == 0x7f;
                            }
                            if (odd && r0 + r >= U.base) atomicOr(&odd_rows[slot * 4 + (r >> 5)], 1u << (r & 31));
                        }
                        asm volatile("bar.sync 2, 128;" ::: "memory");
                    }
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const int id = j * 128 + ptid, r = id / G::CPR, ch = id % G::CPR;
                        uint4 x = v[j];
                        if (careful && (odd_rows[slot * 4 + (r >> 5)] >> (r & 31) & 1)) x = make_uint4(0u, 0u, 0u, 0u);
                        unsigned char* to = smem + (dst - sbase) + r * 128;
                        if constexpr (DT != 2) {
                            *reinterpret_cast<uint4*>(to + (ch >> 3) * G::PANEL + (((ch & 7) ^ (r & 7)) << 4)) = x;
                        } else {
                            uint32_t a[2], b[2], e[2], f[2];
                            Elem<2>::expand(x.x, a);
                            Elem<2>::expand(x.y, b);
                            Elem<2>::expand(x.z, e);
                            Elem<2>::expand(x.w, f);
                            const int c0 = ch * 2;
                            to += (c0 >> 3) * G::PANEL;
                            *reinterpret_cast<uint4*>(to + (((c0 & 7) ^ (r & 7)) << 4)) = make_uint4(a[0], a[1], b[0], b[1]);
                            *reinterpret_cast<uint4*>(to + ((((c0 + 1) & 7) ^ (r & 7)) << 4)) = make_uint4(e[0], e[1], f[0], f[1]);
                        }
                    }
                }
                if constexpr (DT == 2) {
                    signal(c);
                } else {
                    cp_async_commit();
                    if (c >= uint32_t(kWideLag)) {
                        cp_async_wait<kWideLag>();
                        signal(c - kWideLag);
                    }
                }
            }
            wide_next(sh, U, upb);
        }
        if constexpr (DT != 2) {
            cp_async_wait<0>();
            if (ok)
                for (uint32_t k = c > uint32_t(kWideLag) ? c - kWideLag : 0; k < c; ++k) signal(k);
        }
    } else if (w == 12) {
        // ------------------------------------------------------------------ the products
        constexpr uint32_t id_qk = mma_idesc(DT == 0, false, kWideTile), id_pv = mma_idesc(DT == 0, true, D);
        uint32_t c0 = 0;                       // first load of the unit
        uint32_t np[2] = {0, 0}, nq = 0;       // probabilities and units waited for
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (ok && !mbar_wait_bounded(bar, parity)) {
                if (lane == 0) record_status(P.status, ST_ETIMEOUT, blockIdx.x);
                ok = false;
            }
            tm_fence_after();
            return ok;
        };
        auto wait_load = [&](uint32_t l) { return wait(b_full + 8 * ((c0 + l) % G::NS), ((c0 + l) / G::NS) & 1); };
        auto slot_of = [&](uint32_t l) { return s_ring + ((c0 + l) % G::NS) * G::SLOT; };
        auto qk = [&](int s, uint32_t l) {
            if (lane == 0) {
                const uint32_t q = s_q + (MT == 2 ? s * G::SLOT : 0), k = slot_of(l);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t o = (ks >> 2) * G::PANEL + (ks & 3) * 32;
                    mma_ss(tm + s * 128, smem_desc(q + o, 16), smem_desc(k + o, 16), id_qk, ks != 0);
                }
                tm_commit(b_s + 8 * s);
            }
            __syncwarp();
        };
        auto pv = [&](int s, uint32_t l) {
            if (lane == 0) {
                const uint32_t v = slot_of(l);
#pragma unroll
                for (int ks = 0; ks < kWideTile / 16; ++ks)
                    mma_ts(tm + kO + s * D, tm + s * 128 + ks * 8, smem_desc(v + ks * 2048, G::PANEL), id_pv);
            }
            __syncwarp();
        };
        auto release = [&](uint32_t l) {
            if (lane == 0) tm_commit(b_empty + 8 * ((c0 + l) % G::NS));
            __syncwarp();
        };
        auto done = [&](int s) {
            if (lane == 0) tm_commit(b_o + 8 * s);
            __syncwarp();
        };
        for (; ok && sh.pos < sh.end;) {
            const WideUnit U = wide_unit<G>(P, sh);
            const int n = U.n;
            if (!wait(b_q, nq++ & 1)) break;
            if (MT == 2) {
                if (!wait_load(0)) break;
                qk(0, 0);
                qk(1, 0);
                release(0);
                for (int i = 0; i < n; ++i) {
                    if (!wait_load(2 * i + 1)) break;
                    for (int s = 0; s < 2; ++s) {
                        if (!wait(b_p + 8 * s, np[s]++ & 1)) break;
                        pv(s, 2 * i + 1);
                        if (s == 1) release(2 * i + 1);
                        if (i + 1 < n) {
                            if (s == 0 && !wait_load(2 * i + 2)) break;
                            qk(s, 2 * i + 2);
                            if (s == 1) release(2 * i + 2);
                        } else {
                            done(s);
                        }
                    }
                    if (!ok) break;
                }
            } else {
                for (int i = 0; i < min(n, 2); ++i) {
                    if (!wait_load(load_of_k<1>(i))) break;
                    qk(i, load_of_k<1>(i));
                    release(load_of_k<1>(i));
                }
                for (int i = 0; ok && i < n; ++i) {
                    const int s = i & 1;
                    if (!wait_load(load_of_v<1>(i, n))) break;
                    if (!wait(b_p + 8 * s, np[s]++ & 1)) break;
                    pv(s, load_of_v<1>(i, n));
                    release(load_of_v<1>(i, n));
                    if (i + 2 < n) {
                        if (!wait_load(load_of_k<1>(i + 2))) break;
                        qk(s, load_of_k<1>(i + 2));
                        release(load_of_k<1>(i + 2));
                    } else {
                        done(s);
                    }
                }
            }
            c0 += 2 * n;
            wide_next(sh, U, upb);
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
        for (; sh.pos < sh.end;) {
            const WideUnit U = wide_unit<G>(P, sh);
            const int mine = (MT == 2 ? U.n : (U.n - s + 1) / 2);  // steps of this stream
            const int mu = (MT == 2 ? s * kWideTile : 0) + m;      // this thread's query row in the unit
            const int row = U.m0 + mu, t = row / P.G;
            const bool there = mu < U.mrows;
            // query row -> swizzled shared memory (with MT = 1 the two groups take half of the chunks each)
            float f = 1.f;
            {
                const uint16_t* q = P.Q + (long long)sh.b * P.q_sb + (long long)t * P.q_st + (long long)(U.h * P.G + row % P.G) * P.q_sh;
                if (DT == 2) {
                    float top = 0.f;
                    if (there)
                        for (int d = 0; d < D; d += 8) {
                            const uint4 v = __ldg(reinterpret_cast<const uint4*>(q + d));
                            const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) top = fmaxf(top, fmaxf(fabsf(Elem<0>::lo(x[k])), fabsf(Elem<0>::hi(x[k]))));
                        }
                    const int e = (__float_as_int(top) >> 23) & 255;
                    if (e > 0 && e < 255) f = __int_as_float(min(262 - e, 254) << 23);
                }
                for (int ch = MT == 2 ? 0 : s; ch < D / 8; ch += MT == 2 ? 1 : 2) {
                    uint4 v = there ? __ldg(reinterpret_cast<const uint4*>(q + ch * 8)) : make_uint4(0u, 0u, 0u, 0u);
                    if (DT == 2) {
                        uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[k] = MmaHalf::pack(Elem<0>::lo(x[k]) * f, Elem<0>::hi(x[k]) * f);
                        v = make_uint4(x[0], x[1], x[2], x[3]);
                    }
                    *reinterpret_cast<uint4*>(smem + (MT == 2 ? s * G::SLOT : 0) + (ch >> 3) * G::PANEL + m * 128 + (((ch & 7) ^ (m & 7)) << 4)) = v;
                }
            }
            const float scl = P.scale_log2 / f;
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
            fence_proxy_async();
            tm_fence_before();
            __syncwarp();
            if (lane == 0 && ok) mbar_arrive(b_q);

            float ref = -INFINITY, sum = 0.f;
            for (int k = 0; k < mine; ++k) {
                const int i = MT == 2 ? k : 2 * k + s, r0 = (U.tile0 + i) * kWideTile;
                wait(b_s + 8 * s, ns++ & 1);
                const bool draft = U.masked && r0 + kWideTile > U.base;
                const bool hidden = draft || r0 + kWideTile > U.lim;
                // which of 32 rows from r on this query row sees
                auto seen32 = [&](int r) -> uint32_t {
                    uint32_t see = r >= U.lim ? 0u : U.lim - r >= 32 ? ~0u : (1u << (U.lim - r)) - 1;
                    if (draft && r + 32 > U.base) {
                        const int j = r - U.base;  // drafted rows j ..
                        const uint32_t word = j >= 64 ? 0u : j >= 0 ? uint32_t(bits >> j) : (j > -32 ? uint32_t(bits << -j) | ((1u << -j) - 1) : ~0u);
                        see &= word;
                    }
                    return see;
                };
                // the largest logit first: scores are read twice, registers hold 64 of them
                float top = -INFINITY;
                uint32_t a[32], b[32];
                tm_ld32(a, t_s);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t (&x)[32] = (q & 1) ? b : a;
                    tm_wait_ld(x);
                    if (q < 3) tm_ld32((q & 1) ? a : b, t_s + 32 * (q + 1));
                    if (hidden) {
                        const uint32_t see = seen32(r0 + 32 * q);
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (see >> e & 1) top = fmaxf(top, __uint_as_float(x[e]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) top = fmaxf(top, fmaxf(__uint_as_float(x[e]), __uint_as_float(x[e + 1])));
                    }
                }
                top = top * scl - X::kRefShift;
                // the reference moves only when a probability would pass 2^6 of what it was scaled for
                const bool first = ref == -INFINITY, grew = top > ref + 6.f || (first && top > -INFINITY);
                if (__any_sync(~0u, grew && !first)) {
                    const float r = grew ? top : ref, g = grew && !first ? ex2(ref - r) : 1.f;
                    sum *= g;
                    ref = r;
#pragma unroll
                    for (int d = 0; d < D; d += 32) {
                        tm_ld32(a, t_o + d);
                        tm_wait_ld(a);
#pragma unroll
                        for (int e = 0; e < 32; ++e) a[e] = __float_as_uint(__uint_as_float(a[e]) * g);
                        tm_st32(t_o + d, a);
                    }
                } else if (grew) {
                    ref = top;
                }
                const float at = ref == -INFINITY ? 0.f : ref;
                if (draft) {
                    // drafted rows that are not finite went into the tile as zeros: add them for those who see them
                    const uint32_t l = c0 + load_of_v<MT>(i, U.n);
                    wait(b_full + 8 * (l % G::NS), (l / G::NS) & 1);
                    for (int q = 0; q < 4; ++q) {
                        uint32_t odd = ok ? odd_rows[l % G::NS * 4 + q] : 0u;
                        for (; odd; odd &= odd - 1) {
                            const int e = __ffs(int(odd)) - 1, r = r0 + 32 * q + e;
                            const float z = __uint_as_float(tm_read1(t_s + 32 * q + e));
                            const bool see = seen32(r0 + 32 * q) >> e & 1;
                            const float p = see ? ex2(z * scl - at) : 0.f;
                            const uint8_t* v = P.V + attend_offset(P, sh.b, U.h, r & ~15) + (long long)(r & 15) * P.ss;
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
                float part[4] = {0.f, 0.f, 0.f, 0.f};
                tm_ld32(a, t_s);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t (&x)[32] = (q & 1) ? b : a;
                    tm_wait_ld(x);
                    if (q < 3) tm_ld32((q & 1) ? a : b, t_s + 32 * (q + 1));
                    const uint32_t see = hidden ? seen32(r0 + 32 * q) : ~0u;
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float p0 = ex2(fmaf(__uint_as_float(x[e]), scl, -at)), p1 = ex2(fmaf(__uint_as_float(x[e + 1]), scl, -at));
                        if (hidden) {
                            p0 = see >> e & 1 ? p0 : 0.f;
                            p1 = see >> (e + 1) & 1 ? p1 : 0.f;
                        }
                        part[e & 2] += p0;
                        part[(e & 2) + 1] += p1;
                        p[e / 2] = X::pack(p0, p1);
                    }
                    tm_st16(t_s + 16 * q, p);
                }
                sum += (part[0] + part[1]) + (part[2] + part[3]);
                tm_wait_st();
                tm_fence_before();
                __syncwarp();
                if (lane == 0 && ok) mbar_arrive(b_p + 8 * s);
            }
            if (mine > 0) wait(b_o + 8 * s, no++ & 1);

            // ---- the unit's result
            const long long g0 = sh.first + (long long)U.u * U.seq.tiles;
            const long long first_cta = g0 / sh.per_cta, last_cta = (g0 + U.seq.tiles - 1) / sh.per_cta;
            const bool shared = first_cta != last_cta;
            float* part = P.partials + (2ll * blockIdx.x + (first_cta == (long long)blockIdx.x ? 1 : 0)) * G::PSIZE + (MT == 2 ? s * kWideTile * (D + 2) : 0);
            float mref = ref, msum = sum, f_own = 1.f, f_other = 1.f;
            if (MT == 1) {  // join the streams: stream 1 hands its O over, 64 channels at a time
                float2* ml = reinterpret_cast<float2*>(exch);
                ml[s * kWideTile + m] = make_float2(ref, sum);
                named_bar_sync(1, 256);
                const float2 o = ml[(s ^ 1) * kWideTile + m];
                named_bar_sync(1, 256);
                mref = fmaxf(ref, o.x);
                f_own = ref == -INFINITY ? (sum == 0.f ? 0.f : 1.f) : ex2(ref - mref);
                f_other = o.x == -INFINITY ? (o.y == 0.f ? 0.f : 1.f) : ex2(o.x - mref);
                msum = s == 0 ? sum * f_own + o.y * f_other : 0.f;
            }
            const bool writes = there && ok && (MT == 2 || s == 0);
#pragma unroll
            for (int d0 = 0; d0 < D; d0 += 64) {
                constexpr int kHalf = 64;
                const int nd = D - d0 < kHalf ? D - d0 : kHalf;
                if (MT == 1 && s == 1) {
#pragma unroll
                    for (int d = 0; d < nd; d += 32) {
                        uint32_t a[32];
                        tm_ld32(a, t_o + d0 + d);
                        tm_wait_ld(a);
#pragma unroll
                        for (int e = 0; e < 32; ++e) exch[(d + e) * kWideTile + m] = __uint_as_float(a[e]) * f_own;
                    }
                }
                if (MT == 1) named_bar_sync(1, 256);
                if (MT == 2 || s == 0) {
#pragma unroll
                    for (int d = 0; d < nd; d += 32) {
                        uint32_t a[32];
                        tm_ld32(a, t_o + d0 + d);
                        tm_wait_ld(a);
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            float o[4];
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                o[x] = __uint_as_float(a[e + x]) * f_own;
                                if (MT == 1) o[x] += exch[(d + e + x) * kWideTile + m];
                            }
                            if (writes) {
                                if (shared) {
                                    __stcg(reinterpret_cast<float4*>(part + m * D + d0 + d + e), make_float4(o[0], o[1], o[2], o[3]));
                                } else {
                                    attend_write<D, DT>(P, sh.b, U.h, 0, U.m0, U.seq.tokens, mu, d0 + d + e, o, mref, msum);
                                }
                            }
                        }
                    }
                }
                if (MT == 1) named_bar_sync(1, 256);
            }
            if (shared) {
                if (writes) __stcg(reinterpret_cast<float2*>(part + kWideTile * D + 2 * m), make_float2(mref, msum));
                __threadfence();
                named_bar_sync(1, 256);
                const long long unit = (long long)sh.b * upb + U.u;
                if (tid == 0) {
                    *slast = 0;
                    if (ok) {
                        const int n = atomicAdd(P.counters + unit, 1);
                        *slast = n == int(last_cta - first_cta);
                        if (*slast) P.counters[unit] = 0;
                    }
                }
                named_bar_sync(1, 256);
                if (*slast) {
                    __threadfence();
                    for (int x = 0; x < MT; ++x) {
                        const int rows = min(kWideTile, U.mrows - x * kWideTile);
                        attend_combine<D, DT, kWideTile>(P, sh.b, U.h, 0, U.m0 + x * kWideTile, rows, U.seq.tokens, first_cta, last_cta, G::PSIZE,
                                                         x * kWideTile * (D + 2), tid, 256);
                    }
                }
                named_bar_sync(1, 256);
            }
            c0 += 2 * U.n;
            wide_next(sh, U, upb);
        }
    }
    tm_fence_before();
    __syncthreads();
    if (w == 12) tm_free(tm);
}

}  // namespace lagkv
