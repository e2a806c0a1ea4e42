// Attention over a cache held in 8 bits with a scale for each block of rows and head -- sm_100a device code.
//
// The mathematics and the shares of the work are those of lagkv_attend_kernel, over rows k_r = s_K[block of r] c_r
// and v_r = s_V[block of r] d_r with 8-bit codes c, d (int8 or e4m3, both exact in fp16):
//     x_r = scale * log2(e) * s_K * (q . c_r)   (capped: cap * tanh(x / cap)),   p_r = 2^(x_r - ref),
//     out = sum (p_r s_V) d_r / sum p_r.
// K scales enter the fp32 logits.  V scales enter the probabilities before these are rounded to fp16 (half a
// step, 2^-11 of the value at most, like the rounding of a probability anywhere here), relative to a power of two 2^ve that follows the largest scale seen,
// so that the rounded values lie where fp16 is finest whatever the scales.
//
// The products are transposed against lagkv_attend_kernel's: S^T[rows x queries] = C Q^T and O^T[channels x queries] =
// D^T P^T with m16n8k16, rows or channels along M and the query rows of a KV head along N, in groups of eight:
// a decode step of up to 8 query heads per KV head wastes no half of the tensor cores and half of the accumulators.
// Both code operands come straight out of shared memory with 16-byte loads: which channel or row stands for which index
// of a product is free as long as both sides agree.  A word of four channels of one row is two fragments of a
// score product; words of two rows, their bytes paired, are two of an output product.  Probabilities get from the layout of results to
// that of operands by movmatrix.
// Bound by HBM: a tile of 32 rows of 128 channels (8 KB) costs a warp some 300 instructions (e4m3) or 480 (int8).  One token,
// 32 x 8 heads of up to 32768 int8 rows of 128 channels: 265 us, 95 % of the copy rate; 16 x 4 heads of up to 16384 rows in pages of 64:
// 44 us where the bytes take 31.5, the rest is start, tail and joining.  Units of 16 and 32 query rows: bound by issue, 6 x 4
// heads of up to 16411 rows of 64 channels under 35 capped query rows, three units of 16, 46 to 51 us (bytes 6.1).
//
// Calls of few units (a user or two) take the form with a cluster of CTAs for each unit, which join what they have found through
// distributed shared memory: one launch, no partials in memory (1 x 8 x 1216 int8 rows 7.4 us instead of 9.1).
#pragma once
#include <cooperative_groups.h>

#include "lagkv_attend_kernels.cuh"
#include "lagkv_quant_kernels.cuh"

namespace lagkv {

struct QuantAttendParams : AttendParams {  // K, V: codes; block_shift: rows of a scale's block
    const float* K_scale;  // [B, H, blocks]
    const float* V_scale;
    long long blocks;
    float cap_log2, cap_inv;  // cap * log2(e) and its inverse; 0: no cap
    int half;                 // queries and output are fp16 (else bf16)
};

// Two halves of a pair of fp16 from two bytes each.
template <int FORM>
struct Code {  // int8
    // bytes 0 and 2, bytes 1 and 3: 0x6400 | (c + 128) is 1152 + c in fp16
    static __device__ __forceinline__ void widen(uint32_t w, uint32_t& even, uint32_t& odd) {
        uint32_t a, b;
        asm("lop3.b32 %0, %1, 0x00ff00ff, 0x64806480, 0x6a;" : "=r"(a) : "r"(w));
        asm("lop3.b32 %0, %1, 0x00ff00ff, 0x64806480, 0x6a;" : "=r"(b) : "r"(w >> 8));
        asm("sub.f16x2 %0, %1, %2;" : "=r"(even) : "r"(a), "r"(0x64806480u));
        asm("sub.f16x2 %0, %1, %2;" : "=r"(odd) : "r"(b), "r"(0x64806480u));
    }
    static constexpr uint32_t kPairs = 0x5410, kPairsHigh = 0x7632;  // bytes 0, 1 (2, 3) of two words, for widen()
    static __device__ __forceinline__ uint32_t nan_bytes(uint32_t) { return 0u; }
};
template <>
struct Code<FORM_E4M3> {  // bytes 0 and 1, bytes 2 and 3
    static __device__ __forceinline__ void widen(uint32_t w, uint32_t& even, uint32_t& odd) {
        asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }"
            : "=r"(even), "=r"(odd)
            : "r"(w));
    }
    static constexpr uint32_t kPairs = 0x5140, kPairsHigh = 0x7362;
    // 0xff for every byte that is a NaN
    static __device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu); }
};

template <int D_, int FORM_, int NQ_>
struct QuantGeo {
    static constexpr int D = D_, FORM = FORM_, NQ = NQ_;
    static constexpr int NW = kAttendWarps, NT = NW * 32;
    static constexpr int MR = 8 * NQ;                   // query rows of a unit
    static constexpr int MT = D == 256 ? 1 : 2, R = 16 * MT;  // rows of a warp's tile
    static constexpr int CPR = D / 16, KS = D / 16, VW = D / 32;  // 16-byte pieces, score products, words of V a lane holds of a row
    static constexpr int TENSOR = R * D;
    static constexpr int STAGE = 2 * TENSOR + 32;       // and the scales of its groups of 16 rows: K, K, V, V
    static constexpr int FIT = 100 * 1024 / (NW * STAGE), STAGES = FIT > 6 ? 6 : FIT;
    static constexpr int RING = NW * STAGES * STAGE;
    static constexpr int EPI = NW * MR * (D + 4) * 4;   // the warps' accumulators, over the ring
    static constexpr int OFF_JOIN = EPI;                // behind them: what a CTA of a cluster has found
    static constexpr bool QREG = KS * NQ <= 16;         // queries stay in registers, else in shared memory
    static constexpr int OFF_Q = (RING > EPI ? RING : EPI) + 127 & ~127;
    static constexpr int OFF_MASK = OFF_Q + (QREG ? 0 : NQ * KS * 32 * 8);
    static constexpr int OFF_ML = OFF_MASK + MR * 8;    // [NW][MR] reference and sum
    static constexpr int OFF_SCALE = OFF_ML + NW * MR * 8;
    static constexpr int OFF_SCAN = OFF_SCALE + MR * 4;
    static constexpr int SMEM = OFF_SCAN + 64 + 8 * NW;
    static constexpr int CTAS = 2;
    static_assert(EPI + MR * D * 4 + MR * 8 <= RING, "the join lies over the ring, too");
    static_assert(STAGES >= 2 && CTAS * (SMEM + 1024) <= 228 * 1024, "does not fit");

    // Where 16-byte piece c of row r lies in a tile: pieces that eight lanes read together lie in different banks.
    static __device__ __forceinline__ int k_at(int r, int c) { return r * D + ((D >= 128 ? c ^ (r & 1) << 2 : c) << 4); }
    static __device__ __forceinline__ int v_at(int r, int c) {
        if (D >= 128) return r * D + ((c ^ (r & 6)) << 4);
        if (D == 64) return (r >> 1) * 128 + (((r & 1) * 4 + c ^ (r & 6)) << 4);  // two rows to 128 bytes
        return r * D + (c << 4);
    }
    // First channel of word i that lane (g, t) holds of a K row, and of word w of a V row.
    static __device__ __forceinline__ int k_channel(int t, int i) { return D == 96 ? 24 * t + 4 * i : 64 * (i >> 2) + 16 * t + 4 * (i & 3); }
    static __device__ __forceinline__ int v_channel(int g, int w) {
        return D == 96 ? 12 * g + 4 * w : D == 64 ? 8 * g + 4 * w : 128 * (w >> 2) + 16 * g + 4 * (w & 3);
    }
    static __device__ __forceinline__ void load_k(uint32_t (&x)[KS], const unsigned char* tile, int r, int t) {
        if constexpr (D == 96) {
#pragma unroll
            for (int j = 0; j < KS / 2; ++j) *reinterpret_cast<uint2*>(&x[2 * j]) = *reinterpret_cast<const uint2*>(tile + r * D + 24 * t + 8 * j);
        } else {
#pragma unroll
            for (int j = 0; j < KS / 4; ++j) {
                const uint4 v = *reinterpret_cast<const uint4*>(tile + k_at(r, 4 * j + t));
                x[4 * j] = v.x;
                x[4 * j + 1] = v.y;
                x[4 * j + 2] = v.z;
                x[4 * j + 3] = v.w;
            }
        }
    }
    static __device__ __forceinline__ void load_v(uint32_t (&x)[VW], const unsigned char* tile, int r, int g) {
        if constexpr (D == 96) {
#pragma unroll
            for (int w = 0; w < VW; ++w) x[w] = *reinterpret_cast<const uint32_t*>(tile + r * D + 12 * g + 4 * w);
        } else if constexpr (D == 64) {
            const uint2 v = *reinterpret_cast<const uint2*>(tile + v_at(r, g >> 1) + (g & 1) * 8);
            x[0] = v.x;
            x[1] = v.y;
        } else {
#pragma unroll
            for (int j = 0; j < VW / 4; ++j) {
                const uint4 v = *reinterpret_cast<const uint4*>(tile + v_at(r, 8 * j + g));
                x[4 * j] = v.x;
                x[4 * j + 1] = v.y;
                x[4 * j + 2] = v.z;
                x[4 * j + 3] = v.w;
            }
        }
    }
};

__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool full) {
    const int n = full ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {  // an 8 x 8 matrix of 16-bit values
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// tanh without a branch (the instructions on tensor memory need warps that are together), off by 2^-22 at most: below 3/8 the
// series y - y^3 / 3 + 2 y^5 / 15 - 17 y^7 / 315 + 62 y^9 / 2835 (2^-20.9 of tanh y at 3/8, less below), above it 1 - 2 / (1 + e^2y), where
// 2^-22 of e^2y count for less than half and the reciprocal for 2^-23.
__device__ __forceinline__ float quant_tanh(float y) {
    const float a = fabsf(y), q = y * y;
    const float low = y * fmaf(q, fmaf(q, fmaf(q, fmaf(q, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + ex2(a * 2.885390081777927f)));
    return a < 0.375f ? low : copysignf(fmaf(-2.f, r, 1.f), y);
}
__device__ __forceinline__ float pow2_of(int e) { return __int_as_float((e + 127) << 23); }  // -126 <= e <= 127

// The factor that brings a row of bf16 queries with largest magnitude `top` to [2^8, 2^9); 1 where there is none.
__device__ __forceinline__ float quant_query_factor(float top) {
    const int e = (__float_as_int(top) >> 23) & 255;
    return e > 0 && e < 255 ? __int_as_float(min(262 - e, 254) << 23) : 1.f;
}

constexpr float kQuantShift = 8.f;   // a largest probability counts 2^8 ...
constexpr float kQuantSlack = 3.f;   // ... up to 2^11 before the reference follows, and
constexpr int kQuantRange = 4;       // V scales up to 2^4 times 2^ve before that follows: 2^15 fits fp16

template <int D, int FORM, int NQ, bool CLUSTER>
__global__ void __launch_bounds__(kAttendWarps * 32, QuantGeo<D, FORM, NQ>::CTAS)
lagkv_attend_quant_kernel(const __grid_constant__ QuantAttendParams P) {
    using G = QuantGeo<D, FORM, NQ>;
    using C = Code<FORM>;
    constexpr int KS = G::KS, VW = G::VW, MT = G::MT, R = G::R;
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t sbase = smem_u32(smem);
    uint2* sq = reinterpret_cast<uint2*>(smem + G::OFF_Q);
    unsigned long long* smask = reinterpret_cast<unsigned long long*>(smem + G::OFF_MASK);
    float2* sml = reinterpret_cast<float2*>(smem + G::OFF_ML);
    float* sscale = reinterpret_cast<float*>(smem + G::OFF_SCALE);
    long long* sscan = reinterpret_cast<long long*>(smem + G::OFF_SCAN);

    const int upb = P.H * P.mtiles;
    AttendShare sh;
    unsigned rank = 0, ranks = 1;  // CTAs of the unit's cluster
    if constexpr (CLUSTER) {
        const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
        rank = cluster.block_rank();
        ranks = cluster.num_blocks();
        sh.b = int(blockIdx.x / ranks) / upb;
        sh.pos = 0;
        sh.end = 1;
    } else {
        // the joining kernel comes up beside the tail and waits for the partials: 43.3 us instead of 43.8 for the pages above
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        sh = attend_share<G::NT>(P, upb, sscan);
    }
    while (sh.pos < sh.end) {
        AttendSeq seq;
        AttendPart part_of;
        int u, vrow0, vrows;
        if constexpr (CLUSTER) {
            u = int(blockIdx.x / ranks) % upb;
            seq = attend_seq(P, sh.b, u == 0 && rank == 0 && tid == 0);
            const int all = seq.tokens == 0 ? 0 : (seq.len + R - 1) / R;
            vrow0 = int((long long)all * rank / ranks) * R;
            vrows = min(int((long long)all * (rank + 1) / ranks) * R, seq.tokens == 0 ? 0 : seq.len) - vrow0;
        } else {
            seq = attend_seq(P, sh.b, false);
            part_of = attend_part(P, sh, seq.tiles);
            if (part_of.n == 0) {
                attend_advance(P, sh, part_of.step, seq.tiles, upb);
                continue;
            }
            u = part_of.u;
            vrow0 = part_of.tile0 * kAttendTile;
            vrows = max(0, min(part_of.n * kAttendTile, (seq.tokens == 0 ? 0 : seq.len) - vrow0));
        }
        const int m0 = u % P.mtiles * G::MR, h = u / P.mtiles, mrows = min(G::MR, P.T * P.G - m0);
        const int lim = seq.tokens == 0 ? 0 : seq.len, base = seq.len - seq.tokens;
        const bool masked = P.mask != nullptr || seq.tokens > 1;
        const int tiles = (vrows + R - 1) / R;
        const long long scales = ((long long)sh.b * P.H + h) * P.blocks;

        // ---- this warp's tiles w, w + NW, ... ; the first are on their way before anything else
        __syncthreads();  // the ring holds nothing of the unit before
        const int mine = (tiles - w + G::NW - 1) / G::NW;
        // lane l: where group l % MT of 16 rows of this warp's tile (32 / MT) * (i / (32 / MT)) + l / MT lies (-1: not there)
        long long off = -1;
        uint32_t gone = 0, gone_c = 0;  // groups of these without a page
        constexpr int AHEAD = 32 / MT;
        unsigned char* ring = smem + w * G::STAGES * G::STAGE;
        auto issue = [&](int i) {
            if (i < mine) {
                if (i % AHEAD == 0) {
                    off = -1;
                    const int r = vrow0 + (w + (i + lane / MT) * G::NW) * R + lane % MT * 16;
                    const bool wanted = i + lane / MT < mine && r < lim;
                    if (wanted) off = attend_offset(P, sh.b, h, r);
                    gone = __ballot_sync(~0u, wanted && off < 0);
                }
                const int row = vrow0 + (w + i * G::NW) * R;
                const uint32_t dst = smem_u32(ring + (i % G::STAGES) * G::STAGE);
                long long o[MT];
#pragma unroll
                for (int k = 0; k < MT; ++k) o[k] = __shfl_sync(~0u, off, i % AHEAD * MT + k);
#pragma unroll
                for (int j = 0; j < R * G::CPR / 32; ++j) {
                    const int id = j * 32 + lane, r = id / G::CPR, c = id % G::CPR;
                    const long long at = MT == 1 || r < 16 ? o[0] : o[MT - 1];
                    const bool ok = at >= 0 && row + r < lim;
                    const long long src = ok ? at + (long long)(r & 15) * P.ss + c * 16 : 0;
                    cp_async16(dst + G::k_at(r, c), P.K + src, ok);
                    cp_async16(dst + G::TENSOR + G::v_at(r, c), P.V + src, ok);
                }
                if (lane < 2 * MT) {  // 0 for rows that are not there
                    const int k = lane % MT;
                    const bool ok = (MT == 1 || k == 0 ? o[0] : o[MT - 1]) >= 0;
                    const float* s = lane < MT ? P.K_scale : P.V_scale;
                    cp_async4(dst + 2 * G::TENSOR + lane * 4, s + (ok ? scales + ((row + 16 * k) >> P.block_shift) : 0), ok);
                }
            }
            cp_async_commit();
        };
#pragma unroll 1
        for (int i = 0; i < G::STAGES - 1; ++i) issue(i);

        // ---- queries (of query row 8 n + g in lanes g), the factors of their logits, masks
        uint2 q[G::QREG ? NQ : 1][G::QREG ? KS : 1];
        float scl[NQ][2];
        {
            auto load = [&](int n, auto&& put) {  // returns the factor of query row 8 n + g
                const int row = m0 + 8 * n + g;
                const bool there = 8 * n + g < mrows;
                const uint16_t* src = P.Q + (long long)sh.b * P.q_sb + (long long)(row / P.G) * P.q_st + (long long)(h * P.G + row % P.G) * P.q_sh;
                uint2 x[KS];
#pragma unroll
                for (int i = 0; i < KS; ++i) x[i] = there ? __ldg(reinterpret_cast<const uint2*>(src + G::k_channel(t, i))) : make_uint2(0u, 0u);
                float f = 1.f;
                if (!P.half) {
                    float top = 0.f;
#pragma unroll
                    for (int i = 0; i < KS; ++i)
                        top = fmaxf(top, fmaxf(fmaxf(fabsf(Elem<0>::lo(x[i].x)), fabsf(Elem<0>::hi(x[i].x))), fmaxf(fabsf(Elem<0>::lo(x[i].y)), fabsf(Elem<0>::hi(x[i].y)))));
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
                    f = quant_query_factor(top);
#pragma unroll
                    for (int i = 0; i < KS; ++i)
                        x[i] = make_uint2(MmaHalf::pack(Elem<0>::lo(x[i].x) * f, Elem<0>::hi(x[i].x) * f), MmaHalf::pack(Elem<0>::lo(x[i].y) * f, Elem<0>::hi(x[i].y) * f));
                }
#pragma unroll
                for (int i = 0; i < KS; ++i)
                    put(i, FORM == FORM_INT8 ? make_uint2(__byte_perm(x[i].x, x[i].y, 0x5410), __byte_perm(x[i].x, x[i].y, 0x7632)) : x[i]);
                return P.scale_log2 / f;
            };
            if constexpr (G::QREG) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    const float s = load(n, [&](int i, uint2 x) { q[n][i] = x; });
                    scl[n][0] = __shfl_sync(~0u, s, 8 * t);
                    scl[n][1] = __shfl_sync(~0u, s, 8 * t + 4);
                }
            } else {
                for (int n = w; n < NQ; n += G::NW) {
                    const float s = load(n, [&](int i, uint2 x) { sq[(n * KS + i) * 32 + lane] = x; });
                    if (t == 0) sscale[8 * n + g] = s;
                }
            }
            if (tid < G::MR) {
                const int row = m0 + tid, tok = row / P.G;
                unsigned long long bits = 0;
                if (tid < mrows && masked && tok < seq.tokens)
                    bits = P.mask ? P.mask[(long long)sh.b * P.T + tok] : (tok == 63 ? ~0ull : (2ull << tok) - 1);
                smask[tid] = bits;
            }
        }
        __syncthreads();
        if constexpr (!G::QREG) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                scl[n][0] = sscale[8 * n + 2 * t];
                scl[n][1] = sscale[8 * n + 2 * t + 1];
            }
        }

        float acc[2 * VW][NQ][4], ref[NQ][2], sum[NQ][2];
        int ve = -126;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
#pragma unroll
            for (int v = 0; v < 2 * VW; ++v)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[v][n][e] = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                ref[n][e] = -INFINITY;
                sum[n][e] = 0.f;
            }
        }
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
            issue(i + G::STAGES - 1);
            if (i % AHEAD == 0) gone_c = gone;  // issue() is still inside this group of tiles: STAGES <= AHEAD
            cp_async_wait<G::STAGES - 1>();
            __syncwarp();
            const int r0 = vrow0 + (w + i * G::NW) * R;
            const unsigned char* tk = ring + (i % G::STAGES) * G::STAGE;
            const unsigned char* tv = tk + G::TENSOR;
            const float* ts = reinterpret_cast<const float*>(tk + 2 * G::TENSOR);
            const uint32_t miss = gone_c >> (i % AHEAD * MT);  // bit k: group k has no page

            // S^T = C Q^T
            float s[MT][NQ][4];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                uint32_t lo[KS], hi[KS];
                G::load_k(lo, tk, 16 * m + g, t);
                G::load_k(hi, tk, 16 * m + g + 8, t);
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[m][n][e] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    uint32_t a[4];
                    C::widen(lo[k], a[0], a[2]);
                    C::widen(hi[k], a[1], a[3]);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) {
                        const uint2 b = G::QREG ? q[G::QREG ? n : 0][G::QREG ? k : 0] : sq[(n * KS + k) * 32 + lane];
                        MmaHalf::mma(s[m][n], a, b.x, b.y);
                    }
                }
            }

            // softmax step: lane (g, t) has rows g, g + 8 of each group under query rows 2t, 2t + 1 of each eight
            const bool draft = masked && r0 + R > base;
            const bool hidden = r0 + R > lim || draft || (miss & ((1u << MT) - 1));
            float top[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n) top[n][0] = top[n][1] = -INFINITY;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float sk = ts[m];
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[m][n][e] *= scl[n][e & 1] * sk;
            }
            if (P.cap_inv != 0.f) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[m][n][e] = P.cap_log2 * quant_tanh(s[m][n][e] * P.cap_inv);
            }
            if (hidden) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int r = r0 + 16 * m + g + 8 * (e >> 1), j = r - base;
                            bool see = r < lim && !(miss >> m & 1);
                            if (masked && j >= 0) see = see && ((smask[8 * n + 2 * t + (e & 1)] >> (j & 63)) & 1);
                            if (!see) s[m][n][e] = -INFINITY;
                        }
            }
            bool grew = false;
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) top[n][e] = fmaxf(top[n][e], fmaxf(s[m][n][e], s[m][n][e + 2]));
                    grew |= top[n][e] > ref[n][e] + kQuantSlack;  // ref = -infinity: any row that is seen
                }
            float vmax = ts[MT];
            if (MT == 2) vmax = fmaxf(vmax, ts[MT + 1]);
            const int vwant = ((__float_as_int(vmax) >> 23) & 255) - 126;  // vmax < 2^vwant
            const bool wider = vwant > ve + kQuantRange;
            if (__any_sync(~0u, grew) || wider) {
                float back = 1.f;
                if (wider) {
                    const int to = min(vwant, 126);
                    back = ve - to < -126 ? 0.f : pow2_of(ve - to);
                    ve = to;
                }
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    float f[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = top[n][e];
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                        const float now = fmaxf(ref[n][e], x);
                        f[e] = now == -INFINITY ? 1.f : ex2(ref[n][e] - now);
                        ref[n][e] = now;
                        sum[n][e] *= f[e];
                        f[e] *= back;
                    }
#pragma unroll
                    for (int v = 0; v < 2 * VW; ++v)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[v][n][e] *= f[e & 1];
                }
            }
            float at[NQ][2];
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) at[n][e] = ref[n][e] == -INFINITY ? 0.f : ref[n][e] - kQuantShift;

            const float unit = pow2_of(-ve);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float sv = ts[MT + m] * unit;
                uint32_t pb[NQ][2];
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    float p[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[e] = ex2(s[m][n][e] - at[n][e & 1]);
                        sum[n][e & 1] += p[e];
                    }
                    pb[n][0] = transposed(MmaHalf::pack(p[0] * sv, p[1] * sv));
                    pb[n][1] = transposed(MmaHalf::pack(p[2] * sv, p[3] * sv));
                }
                uint32_t x[4][VW];  // rows 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
                for (int k = 0; k < 4; ++k) G::load_v(x[k], tv, 16 * m + 2 * t + (k & 1) + 8 * (k >> 1), g);
                if (FORM == FORM_E4M3 && draft) {
                    // Drafted rows that are NaN must reach the tokens that see them and no others, so not through 0 * NaN:
                    // such codes leave the tile, and the results of those who see them become NaN (all, for rows before the draft).
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int v = 0; v < VW; ++v) x[k][v] &= ~C::nan_bytes(x[k][v]);
#pragma unroll 1
                    for (int r = 0; r < min(16, lim - r0 - 16 * m); ++r) {
                        uint32_t y[VW];
                        G::load_v(y, tv, 16 * m + r, g);
                        bool odd = false;
#pragma unroll
                        for (int v = 0; v < VW; ++v) odd |= C::nan_bytes(y[v]) != 0u;
                        if (!odd) continue;
                        const int j = r0 + 16 * m + r - base;
#pragma unroll
                        for (int n = 0; n < NQ; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                if (j >= 0 && !(smask[8 * n + 2 * t + e] >> (j & 63) & 1)) continue;
#pragma unroll
                                for (int v = 0; v < VW; ++v)
#pragma unroll
                                    for (int c = 0; c < 4; ++c)
                                        if (C::nan_bytes(y[v]) >> (8 * c) & 1) acc[2 * v + (c >> 1)][n][e + 2 * (c & 1)] = __int_as_float(0x7fffffff);
                            }
                    }
                }
                // O^T += D^T P^T: channels c, c + 1 (then c + 2, c + 3) of word v are rows g and g + 8 of a product
#pragma unroll
                for (int v = 0; v < VW; ++v)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t sel = half ? C::kPairsHigh : C::kPairs;
                        uint32_t a[4];
                        C::widen(__byte_perm(x[0][v], x[1][v], sel), a[0], a[1]);
                        C::widen(__byte_perm(x[2][v], x[3][v], sel), a[2], a[3]);
#pragma unroll
                        for (int n = 0; n < NQ; ++n) MmaHalf::mma(acc[2 * v + half][n], a, pb[n][0], pb[n][1]);
                    }
            }
            __syncwarp();
        }
        cp_async_wait<0>();
        __syncthreads();  // the rings are idle: the warps' accumulators go there

        float* epi = reinterpret_cast<float*>(smem) + w * G::MR * (D + 4);
        const float unit = pow2_of(ve);
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float all = sum[n][e];
                all += __shfl_xor_sync(~0u, all, 4);
                all += __shfl_xor_sync(~0u, all, 8);
                all += __shfl_xor_sync(~0u, all, 16);
                const int m = 8 * n + 2 * t + e;
                if (g == 0) sml[w * G::MR + m] = make_float2(ref[n][e] - kQuantShift, all);
#pragma unroll
                for (int v = 0; v < VW; ++v)
                    *reinterpret_cast<float4*>(epi + m * (D + 4) + G::v_channel(g, v)) =
                        make_float4(acc[2 * v][n][e] * unit, acc[2 * v][n][e + 2] * unit, acc[2 * v + 1][n][e] * unit, acc[2 * v + 1][n][e + 2] * unit);
            }
        __syncthreads();

        auto write = [&](int m, int d, const float (&o)[4], float high, float total) {
            if (P.half)
                attend_write<D, 1>(P, sh.b, h, 0, m0, seq.tokens, m, d, o, high, total);
            else
                attend_write<D, 0>(P, sh.b, h, 0, m0, seq.tokens, m, d, o, high, total);
        };
        // four channels of a query row from the warps' accumulators
        auto gather = [&](int m, int d, float (&o)[4], float& high, float& total) {
            high = -INFINITY;
            total = 0.f;
#pragma unroll
            for (int k = 0; k < G::NW; ++k) high = fmaxf(high, sml[k * G::MR + m].x);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = 0.f;
#pragma unroll
            for (int k = 0; k < G::NW; ++k) {
                const float2 ml = sml[k * G::MR + m];
                const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - high);
                if (f == 0.f && ml.y == 0.f) continue;
                total += ml.y * f;
                const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<float*>(smem) + (k * G::MR + m) * (D + 4) + d);
                o[0] += v.x * f;
                o[1] += v.y * f;
                o[2] += v.z * f;
                o[3] += v.w * f;
            }
        };
        if constexpr (CLUSTER) {
            const cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
            float* own = reinterpret_cast<float*>(smem + G::OFF_JOIN);                // [MR][D]
            float2* own_ml = reinterpret_cast<float2*>(smem + G::OFF_JOIN + G::MR * D * 4);  // [MR]
            for (int i = tid; i < mrows * (D / 4); i += G::NT) {
                const int m = i / (D / 4), d = (i % (D / 4)) * 4;
                float o[4], high, total;
                gather(m, d, o, high, total);
                *reinterpret_cast<float4*>(own + m * D + d) = make_float4(o[0], o[1], o[2], o[3]);
                if (d == 0) own_ml[m] = make_float2(high, total);
            }
            cluster.sync();
            // all CTAs' parts in the order of their rows
            for (int i = int(rank) * G::NT + tid; i < mrows * (D / 4); i += int(ranks) * G::NT) {
                const int m = i / (D / 4), d = (i % (D / 4)) * 4;
                float o[4] = {0.f, 0.f, 0.f, 0.f}, high = -INFINITY, total = 0.f;
                for (unsigned r = 0; r < ranks; ++r) high = fmaxf(high, cluster.map_shared_rank(own_ml, r)[m].x);
#pragma unroll 4
                for (unsigned r = 0; r < ranks; ++r) {
                    const float2 ml = cluster.map_shared_rank(own_ml, r)[m];
                    const float4 v = *reinterpret_cast<const float4*>(cluster.map_shared_rank(own, r) + m * D + d);
                    const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - high);
                    if (f == 0.f && ml.y == 0.f) continue;
                    total += ml.y * f;
                    o[0] += v.x * f;
                    o[1] += v.y * f;
                    o[2] += v.z * f;
                    o[3] += v.w * f;
                }
                write(m, d, o, high, total);
            }
            cluster.sync();  // nobody's shared memory goes while another reads it
            sh.pos = sh.end;
        } else {
            // who shares this unit: CTAs c0 .. c1
            const long long c0 = part_of.c0, c1 = part_of.c1;
            constexpr int PSIZE = G::MR * (D + 2);
            float* part = P.partials + (2ll * blockIdx.x + (c0 == (long long)blockIdx.x ? 1 : 0)) * PSIZE;
            for (int i = tid; i < mrows * (D / 4); i += G::NT) {
                const int m = i / (D / 4), d = (i % (D / 4)) * 4;
                float o[4], high, total;
                gather(m, d, o, high, total);
                if (c0 == c1) {
                    write(m, d, o, high, total);
                } else {
                    __stcg(reinterpret_cast<float4*>(part + m * D + d), make_float4(o[0], o[1], o[2], o[3]));
                    if (d == 0) __stcg(reinterpret_cast<float2*>(part + G::MR * D + 2 * m), make_float2(high, total));
                }
            }
            // who shares the unit, for the kernel that joins the partials: said once, by the CTA that starts it
            if (tid == 0 && c0 == (long long)blockIdx.x) P.shared[(long long)sh.b * upb + u] = make_int2(int(c0), int(c1));
            attend_advance(P, sh, part_of.step, seq.tiles, upb);
        }
    }
}

template <int D, int FORM, int NQ>
__global__ void __launch_bounds__(kMergeWarps * 32, 4)
lagkv_attend_quant_merge_kernel(const __grid_constant__ QuantAttendParams P) {
    attend_merge<D, 8 * NQ>(P, [&](int b, int h, int t0, int m0, int tokens, int m, int d, const auto& o, float top, float total) {
        if (P.half)
            attend_write<D, 1>(P, b, h, t0, m0, tokens, m, d, o, top, total);
        else
            attend_write<D, 0>(P, b, h, t0, m0, tokens, m, d, o, top, total);
    });
}

}  // namespace lagkv
