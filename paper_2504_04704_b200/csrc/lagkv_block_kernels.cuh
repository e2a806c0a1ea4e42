// Choosing the blocks of rows that a query attends to -- sm_100a device code.
//
// A block is `block_rows` consecutive rows of one (sequence, KV head).  Its bounds are the per-channel
// minimum and maximum of its K rows, in the storage format (no rounding).  For a query q every logit of
// the block is at most  sum_c max(q_c * min_c, q_c * max_c);  a block's score is the largest such bound
// over the query heads of the KV head.  Scores that decide which blocks are read may differ in their last
// bits only, so the choice is that of scores summed in 64 bits.  Nearly all blocks are far from the border,
// though: scores are first summed in 32 bits, with a bound E on how far off they can be, and only blocks
// within 2 E of the border are summed again in 64 (all in 64 bits took 49 us for eight caches of 2048 blocks,
// where the bounds are read in 10).
#pragma once
#include "lagkv_attend_kernels.cuh"

namespace lagkv {

constexpr int kBoundsThreads = 256;
constexpr int kScoreThreads = 128;
constexpr int kScoreHeads = 8;                   // query heads of one pass of matrix products
constexpr int kScoreChunk = 32;                  // blocks that a CTA takes in one go
constexpr int kSelectThreads = 512;
constexpr int kSelectBins = 2048;

// ------------------------------------------------------------------------------------ bounds
// One warp per block: 16-byte loads, a row per group of lanes, packed min / max, groups joined by
// shuffles.  Reads each row once and writes two rows per block: bound by HBM reads.
template <int DT>
__global__ void __launch_bounds__(kBoundsThreads, 3)  // without the 3: spills, 257 us where this takes 246 (1.6 GB)
lagkv_block_bounds_kernel(const AttendParams P, const int32_t* __restrict__ from_len, uint8_t* __restrict__ bounds,
                          long long blocks, int ctas_per_unit, int cpr) {
    using E = Elem<DT>;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const long long unit = blockIdx.x / ctas_per_unit;
    const int b = int(unit / P.H), h = int(unit % P.H);
    const int len = __ldg(P.seq_len + b), from = from_len ? __ldg(from_len + b) : 0;
    if (len < 0 || len > P.S_cap || from < 0) {
        if (h == 0 && blockIdx.x % ctas_per_unit == 0 && threadIdx.x == 0) record_status(P.status, ST_EINVAL, b);
        return;
    }
    const int shift = P.block_shift;
    const int nb = (len + (1 << shift) - 1) >> shift;
    const int rpl = 32 / cpr, c = lane % cpr, rr = lane / cpr;
    const bool active = rr < rpl;
    for (long long j = (from >> shift) + (blockIdx.x % ctas_per_unit) * (kBoundsThreads / 32) + w; j < nb;
         j += (long long)ctas_per_unit * (kBoundsThreads / 32)) {
        uint32_t mn[4 * E::PW], mx[4 * E::PW];
#pragma unroll
        for (int i = 0; i < 4 * E::PW; ++i) {
            mn[i] = E::kPosInf2;
            mx[i] = E::kNegInf2;
        }
        const int r0 = int(j << shift), rows = min(1 << shift, len - r0);
        for (int g = 0; g < rows; g += kWarpRows) {
            const long long off = attend_offset(P, b, h, r0 + g);
            if (off < 0) continue;
            const int n = min(kWarpRows, rows - g);
            const uint8_t* base = P.K + off + c * 16;
            auto take = [&](const uint4& v) {
                const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t p[E::PW];
                    E::expand(word[i], p);
#pragma unroll
                    for (int k = 0; k < E::PW; ++k) {
                        mn[i * E::PW + k] = E::min2(mn[i * E::PW + k], p[k]);
                        mx[i * E::PW + k] = E::max2(mx[i * E::PW + k], p[k]);
                    }
                }
            };
            if (active) {
                // a row index behind the last one repeats the last row: it changes no minimum
                for (int r = rr; r < n; r += 8 * rpl) {
                    uint4 v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i == 0 || i * rpl < kWarpRows) v[i] = __ldg(reinterpret_cast<const uint4*>(base + (long long)min(r + i * rpl, n - 1) * P.ss));
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i == 0 || i * rpl < kWarpRows) take(v[i]);
                }
            }
        }
        for (int s = 1; s < rpl; ++s) {
#pragma unroll
            for (int i = 0; i < 4 * E::PW; ++i) {
                const uint32_t a = __shfl_sync(~0u, mn[i], (c + s * cpr) & 31), z = __shfl_sync(~0u, mx[i], (c + s * cpr) & 31);
                if (rr == 0) {
                    mn[i] = E::min2(mn[i], a);
                    mx[i] = E::max2(mx[i], z);
                }
            }
        }
        if (rr == 0) {
            uint8_t* to = bounds + ((unit * blocks + j) * 2 * cpr + c) * 16;
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (DT == 2) {
                    asm("{ .reg .b16 l, h; cvt.rn.satfinite.e4m3x2.f16x2 l, %1; cvt.rn.satfinite.e4m3x2.f16x2 h, %2; mov.b32 %0, {l, h}; }"
                        : "=r"(lo[i])
                        : "r"(mn[2 * i]), "r"(mn[2 * i + 1]));
                    asm("{ .reg .b16 l, h; cvt.rn.satfinite.e4m3x2.f16x2 l, %1; cvt.rn.satfinite.e4m3x2.f16x2 h, %2; mov.b32 %0, {l, h}; }"
                        : "=r"(hi[i])
                        : "r"(mx[2 * i]), "r"(mx[2 * i + 1]));
                } else {
                    lo[i] = mn[i];
                    hi[i] = mx[i];
                }
            }
            *reinterpret_cast<uint4*>(to) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            *reinterpret_cast<uint4*>(to + cpr * 16) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        }
    }
}

// ------------------------------------------------------------------------------------ scores
// order-preserving map double -> uint64
__device__ __forceinline__ unsigned long long double_key(double f) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(f);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
// pair `p` of channels of a row of bounds, as two floats
template <int DT>
__device__ __forceinline__ f32x2 bound_pair(const uint8_t* row, int p) {
    if constexpr (DT == 2) {
        uint32_t w[2];
        Elem<2>::expand(__ldg(reinterpret_cast<const uint16_t*>(row) + p), w);
        return widen2<Elem<2>>(w[0]);
    } else {
        return widen2<Elem<DT>>(__ldg(reinterpret_cast<const uint32_t*>(row) + p));
    }
}
// pair `p` of channels of a query
template <int DT>
__device__ __forceinline__ f32x2 query_pair(const uint16_t* q, int p) {
    return widen2<Elem<DT == 1 ? 1 : 0>>(__ldg(reinterpret_cast<const uint32_t*>(q) + p));
}
__device__ __forceinline__ float max_of_warp(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

// What one launch of the score kernel looks like.
struct ScoreShape {
    long long blocks;     // blocks per (sequence, KV head) of the bounds
    int chunks, chunk;    // CTAs per unit, blocks per CTA
    float* approx;        // [units][blocks]
    float* error;         // [units][chunks]
};

// With q = q+ + q- (its positive and negative parts) a block's bound is sum q+ max + q- min: a product of 16-bit
// matrices, eight heads by eight blocks a warp.  The order of the channels in a sum is free, so a lane loads
// 16-byte pieces as they lie and both operands meet them in that order.  Products of 16-bit values are exact; each
// of the D additions that are not of zeros is off by at most 2^-23 of sum |q_c| m_c <= |q| |m|, m_c =
// max(|min_c|, |max_c|); E allows twice that.  (Multiply-adds in the lanes and shuffles took 23 us where
// this takes 16, at eight caches of 2048 blocks.)
template <int DT, int D>
__global__ void __launch_bounds__(kScoreThreads)
lagkv_block_score_kernel(const AttendParams P, const uint8_t* __restrict__ bounds, const ScoreShape S) {
    using E = Elem<DT>;
    using X = Mma<DT>;
    constexpr int ROWB = D * E::EB, CPR = ROWB / 16, K = (CPR + 3) / 4, EPC = 16 / E::EB;  // pieces per row and lane, channels per piece
    constexpr int W = 4 * E::PW;                                                            // 16-bit pairs per piece
    __shared__ float red[kScoreThreads / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = lane & 3, row = lane >> 2;
    const long long unit = blockIdx.x / S.chunks;  // (b * T + t) * H + h
    const int h = int(unit % P.H), t = int(unit / P.H % P.T), b = int(unit / P.H / P.T), chunk = int(blockIdx.x % S.chunks);
    const AttendSeq seq = attend_seq(P, b, false);
    if (seq.tokens == 0) return;
    const int lim = seq.len - (P.T - 1 - t), nb = (lim + (1 << P.block_shift) - 1) >> P.block_shift;
    const int j0 = chunk * S.chunk, j1 = min(nb, j0 + S.chunk);
    if (j0 >= nb || nb <= P.keep) return;  // nothing to choose
    const uint8_t* rows = bounds + ((long long)b * P.H + h) * S.blocks * 2 * ROWB;
    float q2 = 0.f, m2 = 0.f;  // largest squared norms
    for (int g0 = 0; g0 < P.G; g0 += kScoreHeads) {
        const bool head = g0 + row < P.G;
        const uint16_t* q = P.Q + (long long)b * P.q_sb + (long long)t * P.q_st + (long long)(h * P.G + min(g0 + row, P.G - 1)) * P.q_sh;
        // this lane's channels of its head, positive and negative parts (fp8: scaled to fp16 by a power of two)
        uint32_t pos[K][W], neg[K][W];
        float n2 = 0.f, back = 1.f, top = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool in = CPR % 4 == 0 || c + 4 * k < CPR;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                pos[k][i] = in ? __ldg(reinterpret_cast<const uint32_t*>(q + (c + 4 * k) * EPC) + i) : 0u;
                const float x = q_to_float(uint16_t(pos[k][i]), DT == 1), y = q_to_float(uint16_t(pos[k][i] >> 16), DT == 1);
                n2 = fmaf(x, x, fmaf(y, y, n2));
                top = fmaxf(top, fmaxf(fabsf(x), fabsf(y)));
            }
        }
        if (DT == 2) {
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
            const int e = (__float_as_int(top) >> 23) & 255;
            const float f = e > 0 && e < 255 ? __int_as_float(min(262 - e, 254) << 23) : 1.f;
            back = 1.f / f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < W; ++i) pos[k][i] = MmaHalf::pack(Elem<0>::lo(pos[k][i]) * f, Elem<0>::hi(pos[k][i]) * f);
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                neg[k][i] = E::min2(pos[k][i], 0u);
                pos[k][i] = E::max2(pos[k][i], 0u);
            }
        n2 += __shfl_xor_sync(~0u, n2, 1);
        n2 += __shfl_xor_sync(~0u, n2, 2);
        q2 = fmaxf(q2, n2 == n2 ? n2 : INFINITY);
        for (int j = j0 + w * 8; j < j1; j += kScoreThreads / 32 * 8) {
            const uint8_t* lo = rows + (long long)min(j + row, nb - 1) * 2 * ROWB;
            uint4 vl[K], vh[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const bool in = CPR % 4 == 0 || c + 4 * k < CPR;
                vl[k] = in ? __ldg(reinterpret_cast<const uint4*>(lo) + c + 4 * k) : make_uint4(0u, 0u, 0u, 0u);
                vh[k] = in ? __ldg(reinterpret_cast<const uint4*>(lo + ROWB) + c + 4 * k) : make_uint4(0u, 0u, 0u, 0u);
            }
            float acc[4] = {0.f, 0.f, 0.f, 0.f}, n = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const uint32_t wl[4] = {vl[k].x, vl[k].y, vl[k].z, vl[k].w}, wh[4] = {vh[k].x, vh[k].y, vh[k].z, vh[k].w};
                uint32_t pl[W], ph[W];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t x[E::PW], y[E::PW];
                    E::expand(wl[i], x);
                    E::expand(wh[i], y);
#pragma unroll
                    for (int e = 0; e < E::PW; ++e) {
                        pl[i * E::PW + e] = x[e];
                        ph[i * E::PW + e] = y[e];
                    }
                }
#pragma unroll
                for (int i = 0; i < W; i += 2) {
                    const uint32_t ap[4] = {pos[k][i], 0u, pos[k][i + 1], 0u}, an[4] = {neg[k][i], 0u, neg[k][i + 1], 0u};
                    X::mma(acc, ap, ph[i], ph[i + 1]);
                    X::mma(acc, an, pl[i], pl[i + 1]);
                }
                if (g0 == 0) {
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const float x = fmaxf(fabsf(E::lo(pl[i])), fabsf(E::lo(ph[i]))), y = fmaxf(fabsf(E::hi(pl[i])), fabsf(E::hi(ph[i])));
                        n = fmaf(x, x, fmaf(y, y, n));
                    }
                }
            }
            // acc[0], acc[1]: head `row`, blocks 2 c and 2 c + 1: the largest over the heads
            float s0 = head ? acc[0] * back : -INFINITY, s1 = head ? acc[1] * back : -INFINITY;
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                s0 = fmaxf(s0, __shfl_xor_sync(~0u, s0, o));
                s1 = fmaxf(s1, __shfl_xor_sync(~0u, s1, o));
            }
            if (lane < 4) {
                float* to = S.approx + unit * S.blocks + j + 2 * c;
                if (j + 2 * c < j1) to[0] = g0 ? fmaxf(to[0], s0) : s0;
                if (j + 2 * c + 1 < j1) to[1] = g0 ? fmaxf(to[1], s1) : s1;
            }
            n += __shfl_xor_sync(~0u, n, 1);
            n += __shfl_xor_sync(~0u, n, 2);
            m2 = fmaxf(m2, n == n ? n : INFINITY);
        }
    }
    // 1.01: the roundings of the norms themselves.  Squares below 2^-149 vanish from them, at most D * 2^-149 in all: next
    // to 2^-100 that is nothing, so smaller norms count as 2^-50.  Products that vanish (D * 2^-126) are covered with it.
    const float e = 1.01f * (D + 16) * 0x1p-22f * sqrtf(fmaxf(max_of_warp(q2), 0x1p-100f)) * sqrtf(fmaxf(max_of_warp(m2), 0x1p-100f));
    if (lane == 0) red[w] = e == e ? e : INFINITY;
    __syncthreads();
    if (threadIdx.x == 0) {
        float top = 0.f;
        for (int i = 0; i < kScoreThreads / 32; ++i) top = fmaxf(top, red[i]);
        S.error[unit * S.chunks + chunk] = top;
    }
}

// ------------------------------------------------------------------------------------ choice
// Narrows [lo, hi] (the smallest and the largest of the keys asked about) around the key with `need` - 1 larger
// ones, by histograms over 2048 bins, until enough(lo, hi) or the interval is one key; leaves in `need` how many
// of the keys in [lo, hi] are wanted, and in `all` whether that is all of them.
template <class Key, class Get, class Enough>
__device__ __forceinline__ void find_border(Key& lo, Key& hi, int n, int& need, bool& all, int* hist, int* wsum, int* found, Get&& get,
                                            Enough&& enough) {
    constexpr int NW = kSelectThreads / 32, PER = kSelectBins / kSelectThreads;
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    for (;;) {
        const int width = sizeof(Key) == 8 ? 64 - __clzll((long long)(hi - lo)) : 32 - __clz(int(hi - lo)), shift = max(0, width - 11);
        __syncthreads();
        for (int i = tid; i < kSelectBins; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kSelectThreads) {
            const Key k = get(j);
            if (k >= lo && k <= hi) atomicAdd(&hist[int((k - lo) >> shift)], 1);
        }
        __syncthreads();
        const int top = kSelectBins - PER * (tid + 1);  // this thread's bins, counted from the top
        int mine = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) mine += hist[top + i];
        int inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(~0u, inc, o);
            if (lane >= o) inc += v;
        }
        if (lane == 31) wsum[w] = inc;
        __syncthreads();
        const int before = inc - mine + __reduce_add_sync(~0u, lane < w && lane < NW ? wsum[lane] : 0);
        if (before < need && before + mine >= need) {
            int at = before;
            for (int i = PER - 1; i >= 0; --i) {
                const int c = hist[top + i];
                if (at + c >= need) {
                    found[0] = top + i;
                    found[1] = need - at;
                    found[2] = c;
                    break;
                }
                at += c;
            }
        }
        __syncthreads();
        const Key new_lo = lo + (Key(found[0]) << shift), span = shift == 0 ? Key(0) : (Key(1) << shift) - 1;
        hi = hi - new_lo < span ? hi : new_lo + span;
        lo = new_lo;
        need = found[1];
        all = found[2] == need;
        if (lo == hi || enough(lo, hi)) return;
    }
}

// The 64-bit bound of one block for one query head, by eight lanes.
template <int DT>
__device__ __forceinline__ double exact_bound(const uint8_t* row, const uint16_t* q0, int D, int rowb, int lane) {
    double sum = 0.0;
#pragma unroll 4
    for (int p = lane; p < D / 2; p += 8) {
        float q[2], lo[2], hi[2];
        unpack2(query_pair<DT>(q0, p), q[0], q[1]);
        unpack2(bound_pair<DT>(row, p), lo[0], lo[1]);
        unpack2(bound_pair<DT>(row + rowb, p), hi[0], hi[1]);
#pragma unroll
        for (int e = 0; e < 2; ++e) sum = fma(double(q[e]), double(q[e] >= 0.f ? hi[e] : lo[e]), sum);
    }
#pragma unroll
    for (int o = 4; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    return sum;
}

// Numbers in order for what the CTA's warps count: v is the warp's count; returns the sum over the warps before it.
__device__ __forceinline__ int warps_before(int v, int* wsum, int& total) {
    constexpr int NW = kSelectThreads / 32;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    __syncthreads();
    if (lane == 0) wsum[w] = v;
    __syncthreads();
    const int x = lane < NW ? wsum[lane] : 0;
    total = __reduce_add_sync(~0u, x);
    return __reduce_add_sync(~0u, lane < w ? x : 0);
}

// One CTA per (sequence, token, KV head): the first `sink` and last `recent` blocks and the best of the
// others, `keep` in all, lower block first among equals, written in ascending order with -1 behind.
template <int DT>
__global__ void __launch_bounds__(kSelectThreads, 2)  // without the 2: 40 registers, spills, 3 us more
lagkv_block_select_kernel(const AttendParams P, const uint8_t* __restrict__ bounds, const ScoreShape S, int D,
                          unsigned long long* __restrict__ keys, int sink, int recent, int32_t* __restrict__ idx) {
    extern __shared__ float sa[];  // the candidates' scores, then the numbers of those near the border
    __shared__ __align__(8) int hist[kSelectBins];
    __shared__ uint32_t ends[2][kSelectThreads / 32];
    __shared__ float errors[kSelectThreads / 32];
    __shared__ int wsum[2][kSelectThreads / 32];
    __shared__ int found[3];
    __shared__ unsigned long long range[2];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    constexpr int NW = kSelectThreads / 32;
    const long long unit = blockIdx.x;
    const int h = int(unit % P.H), t = int(unit / P.H % P.T), b = int(unit / P.H / P.T);
    const AttendSeq seq = attend_seq(P, b, unit % ((long long)P.H * P.T) == 0 && tid == 0);
    const int lim = seq.tokens == 0 ? 0 : seq.len - (P.T - 1 - t);
    const int nb = (lim + (1 << P.block_shift) - 1) >> P.block_shift;
    int32_t* out = idx + unit * P.keep;
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the scores
    if (nb <= P.keep) {
        for (int i = tid; i < P.keep; i += kSelectThreads) out[i] = i < nb ? i : -1;
        return;
    }
    float above = 0.f, below = 0.f, over = 0.f;
    bool near_all = false;
    auto sure = [&](float a) { return a > above + over; };
    auto out_of_it = [&](float a) { return a < below - over; };
    // candidates: blocks [sink, nb - recent); nb > keep >= sink + recent, so there are more than are wanted
    const int n = nb - recent - sink;
    int need = P.keep - sink - recent;
    if (need > 0) {
        uint32_t lo = ~0u, hi = 0u;
        float error = 0.f;
        const float* approx = S.approx + unit * S.blocks + sink;
        for (int j = tid; j < n; j += 4 * kSelectThreads) {  // a block taken twice changes neither end
            float a[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = __ldcg(approx + min(j + i * kSelectThreads, n - 1));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (j + i * kSelectThreads < n) sa[j + i * kSelectThreads] = a[i];
                lo = min(lo, float_key(a[i]));
                hi = max(hi, float_key(a[i]));
            }
        }
        for (int c = tid; c < (nb + S.chunk - 1) / S.chunk; c += kSelectThreads) error = fmaxf(error, __ldcg(S.error + unit * S.chunks + c));
        lo = __reduce_min_sync(~0u, lo);
        hi = __reduce_max_sync(~0u, hi);
        error = max_of_warp(error);
        if (lane == 0) {
            ends[0][w] = lo;
            ends[1][w] = hi;
            errors[w] = error;
        }
        __syncthreads();
        lo = __reduce_min_sync(~0u, ends[0][lane % NW]);
        hi = __reduce_max_sync(~0u, ends[1][lane % NW]);
        error = max_of_warp(errors[lane % NW]);
        bool all;
        int rank = need;
        auto value = [](uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); };
        find_border<uint32_t>(lo, hi, n, rank, all, hist, wsum[0], found, [&](int j) { return float_key(sa[j]); },
                              [&](uint32_t x, uint32_t y) { return value(y) - value(x) <= error; });
        // the need-th largest 32-bit score is in [lo, hi], the need-th largest 64-bit one within E of that
        above = value(hi) + 2.f * error * 1.0001f;
        below = value(lo) - 2.f * error * 1.0001f;
        over = fmaxf(fabsf(value(lo)), fabsf(value(hi))) * 0x1p-22f;  // the two sums above are rounded
        int* near = reinterpret_cast<int*>(sa) + n;
        // blocks near the border, in their order: a warp takes a run of candidates
        const int run = ((n + kSelectThreads - 1) / kSelectThreads) * 32, j0 = min(n, w * run), j1 = min(n, j0 + run);
        int ni = 0, na = 0;
        for (int j = j0 + lane; j < j1; j += 32) {
            ni += sure(sa[j]);
            na += !sure(sa[j]) && !out_of_it(sa[j]);
        }
        int total_in, total_near;
        warps_before(__reduce_add_sync(~0u, ni), wsum[0], total_in);
        int at = warps_before(__reduce_add_sync(~0u, na), wsum[1], total_near);
        int wanted = need - total_in;  // of the blocks near the border; at least one
        near_all = wanted >= total_near;
        if (!near_all) {
            for (int j = j0; j < j1; j += 32) {
                const bool in = j + lane < j1 && !sure(sa[j + lane]) && !out_of_it(sa[j + lane]);
                const uint32_t m = __ballot_sync(~0u, in);
                if (in) near[at + __popc(m & ((1u << lane) - 1))] = j + lane;
                at += __popc(m);
            }
            __syncthreads();
            const int rowb = D * Elem<DT>::EB;
            const uint8_t* rows = bounds + (((long long)b * P.H + h) * S.blocks + sink) * 2 * rowb;
            const uint16_t* q0 = P.Q + (long long)b * P.q_sb + (long long)t * P.q_st + (long long)(h * P.G) * P.q_sh;
            const bool few = total_near <= kSelectThreads;
            unsigned long long* mine = few ? reinterpret_cast<unsigned long long*>(hist) : keys + unit * S.blocks;
            for (int i = tid; i < total_near; i += kSelectThreads) mine[i] = 0ull;
            __syncthreads();
            const int pairs = total_near * P.G;
            for (int i0 = w * 4; i0 < pairs; i0 += NW * 4) {
                const int i = min(i0 + (lane >> 3), pairs - 1), j = i / P.G;  // a pair taken twice changes no maximum
                const double sum = exact_bound<DT>(rows + (long long)near[j] * 2 * rowb, q0 + (long long)(i - j * P.G) * P.q_sh, D, rowb, lane & 7);
                if ((lane & 7) == 0) atomicMax(&mine[j], double_key(sum == sum ? sum : -INFINITY));
            }
            __syncthreads();
            // The chosen ones become certain, the others impossible.  Few are ranked one against another (for the
            // usual handful 1.4 us less than the histograms), many by the histograms.
            if (few) {
                if (tid < total_near) {
                    const unsigned long long k = mine[tid];
                    int above_it = 0;
                    for (int i = 0; i < total_near; ++i) above_it += mine[i] > k || (mine[i] == k && i < tid);
                    sa[near[tid]] = above_it < wanted ? INFINITY : -INFINITY;
                }
            } else {
                if (tid == 0) {
                    range[0] = ~0ull;
                    range[1] = 0ull;
                }
                __syncthreads();
                for (int i = tid; i < total_near; i += kSelectThreads) {
                    atomicMin(&range[0], mine[i]);
                    atomicMax(&range[1], mine[i]);
                }
                __syncthreads();
                unsigned long long k = range[0], k_hi = range[1];
                find_border<unsigned long long>(k, k_hi, total_near, wanted, all, hist, wsum[0], found, [&](int i) { return mine[i]; },
                                                [&](unsigned long long, unsigned long long) { return all; });
                // of keys equal to k the lowest blocks
                const int pn = (total_near + kSelectThreads - 1) / kSelectThreads, i0 = min(total_near, tid * pn), i1 = min(total_near, i0 + pn);
                int ne = 0;
                for (int i = i0; i < i1; ++i) ne += mine[i] == k;
                int ie = ne;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int x = __shfl_up_sync(~0u, ie, o);
                    if (lane >= o) ie += x;
                }
                int all_equal;
                int be = warps_before(__shfl_sync(~0u, ie, 31), wsum[0], all_equal) + ie - ne;
                for (int i = i0; i < i1; ++i) {
                    const bool in = all ? mine[i] >= k : mine[i] > k || (mine[i] == k && be < wanted);
                    be += mine[i] == k;
                    sa[near[i]] = in ? INFINITY : -INFINITY;
                }
            }
            __syncthreads();
        }
    }
    // ordered output: a warp takes a run of blocks
    auto taken = [&](int j) {
        if (j >= nb) return false;
        if (j < sink || j >= sink + n) return true;
        if (need == 0) return false;
        const float a = sa[j - sink];
        return sure(a) || a == INFINITY || (near_all && !out_of_it(a));
    };
    const int run = ((nb + kSelectThreads - 1) / kSelectThreads) * 32, j0 = w * run, j1 = min(nb, j0 + run);
    int c = 0, total;
    for (int j = j0 + lane; j < j1; j += 32) c += taken(j);
    int at = warps_before(__reduce_add_sync(~0u, c), wsum[0], total);
    for (int j = j0; j < j1; j += 32) {
        const bool in = taken(j + lane);
        const uint32_t m = __ballot_sync(~0u, in);
        if (in) out[at + __popc(m & ((1u << lane) - 1))] = j + lane;
        at += __popc(m);
    }
}

}  // namespace lagkv
