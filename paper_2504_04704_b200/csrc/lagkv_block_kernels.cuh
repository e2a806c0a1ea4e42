// Choosing the blocks of rows that a query attends to -- sm_100a device code.
//
// A block is `block_rows` consecutive rows of one (sequence, KV head).  Its bounds are the per-channel
// minimum and maximum of its K rows, in the storage format (no rounding).  For a query q every logit of
// the block is at most  sum_c max(q_c * min_c, q_c * max_c);  a block's score is the largest such bound
// over the query heads of the KV head.  Scores that decide which blocks are read may differ in their last
// bits only, so they are summed in 64 bits: the choice does not depend on the order of the sums.
#pragma once
#include "lagkv_attend_kernels.cuh"

namespace lagkv {

constexpr int kBoundsThreads = 256;
constexpr int kScoreThreads = 128;
constexpr int kScoreBlocks = kScoreThreads / 4;  // blocks per CTA: four lanes each
constexpr int kScoreHeads = 8;                   // query heads whose sums a thread holds at a time
constexpr int kSelectThreads = 256;
constexpr int kSelectBins = 2048;

// ------------------------------------------------------------------------------------ bounds
// One warp per block: 16-byte loads, a row per group of lanes, packed min / max, groups joined by
// shuffles.  Reads each row once and writes two rows per block: bound by HBM reads.
template <int DT>
__global__ void __launch_bounds__(kBoundsThreads)
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

// Four lanes per block, each a quarter of its 16-byte chunks; the queries wait in shared memory in 64
// bits.  Products of 16-bit values are exact, sums are off by less than 2^-45 of the largest term.
template <int DT>
__global__ void __launch_bounds__(kScoreThreads)
lagkv_block_score_kernel(const AttendParams P, const uint8_t* __restrict__ bounds, long long blocks, int chunks, int D,
                         unsigned long long* __restrict__ keys) {
    using E = Elem<DT>;
    constexpr int EPC = 16 / E::EB;  // channels per 16-byte chunk
    extern __shared__ double sq[];   // [kScoreHeads][D + 2]
    const int tid = threadIdx.x, ql = tid & 3;
    const long long unit = blockIdx.x / chunks;  // (b * T + t) * H + h
    const int h = int(unit % P.H), t = int(unit / P.H % P.T), b = int(unit / P.H / P.T);
    const AttendSeq seq = attend_seq(P, b, false);
    if (seq.tokens == 0) return;
    const int lim = seq.len - (P.T - 1 - t), nb = (lim + (1 << P.block_shift) - 1) >> P.block_shift;
    const int j0 = int(blockIdx.x % chunks) * kScoreBlocks;
    if (j0 >= nb || nb <= P.keep) return;  // nothing to choose
    const int j = j0 + (tid >> 2), cpr = D / EPC;
    const uint8_t* lo = bounds + (((long long)b * P.H + h) * blocks + min(j, nb - 1)) * 2 * cpr * 16;
    double best = -INFINITY;
    for (int g0 = 0; g0 < P.G; g0 += kScoreHeads) {
        const int gn = min(kScoreHeads, P.G - g0);
        __syncthreads();
        for (int i = tid; i < kScoreHeads * D; i += kScoreThreads) {
            const int g = i / D, d = i % D;
            float v = 0.f;
            if (g < gn)
                v = q_to_float(__ldg(P.Q + (long long)b * P.q_sb + (long long)t * P.q_st + (long long)(h * P.G + g0 + g) * P.q_sh + d), DT == 1);
            sq[g * (D + 2) + d] = double(v);
        }
        __syncthreads();
        double acc[kScoreHeads];
#pragma unroll
        for (int g = 0; g < kScoreHeads; ++g) acc[g] = 0.0;
        for (int c = ql; c < cpr; c += 4) {
            const uint4 vl = __ldg(reinterpret_cast<const uint4*>(lo) + c), vh = __ldg(reinterpret_cast<const uint4*>(lo) + cpr + c);
            const uint32_t wl[4] = {vl.x, vl.y, vl.z, vl.w}, wh[4] = {vh.x, vh.y, vh.z, vh.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t pl[E::PW], ph[E::PW];
                E::expand(wl[i], pl);
                E::expand(wh[i], ph);
#pragma unroll
                for (int k = 0; k < E::PW; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const double mn = e ? E::hi(pl[k]) : E::lo(pl[k]), mx = e ? E::hi(ph[k]) : E::lo(ph[k]);
                        const double* q = sq + c * EPC + (i * E::PW + k) * 2 + e;
#pragma unroll
                        for (int g = 0; g < kScoreHeads; ++g) {
                            if (g < gn) {
                                const double x = q[g * (D + 2)];
                                acc[g] = fma(x, x >= 0.0 ? mx : mn, acc[g]);
                            }
                        }
                    }
            }
        }
#pragma unroll
        for (int g = 0; g < kScoreHeads; ++g) {
            if (g < gn) {
                acc[g] += __shfl_xor_sync(~0u, acc[g], 1);
                acc[g] += __shfl_xor_sync(~0u, acc[g], 2);
                best = fmax(best, acc[g]);
            }
        }
    }
    if (ql == 0 && j < nb) keys[unit * blocks + j] = double_key(best);
}

// ------------------------------------------------------------------------------------ choice
// One CTA per (sequence, token, KV head): the first `sink` and last `recent` blocks and the best of the
// others, `keep` in all, lower block first among equals, written in ascending order with -1 behind.  The
// border is found by histograms over the range of the keys, each pass narrowing it to one of 2048 bins.
__global__ void __launch_bounds__(kSelectThreads)
lagkv_block_select_kernel(const AttendParams P, const unsigned long long* __restrict__ keys, long long blocks, int sink,
                          int recent, int32_t* __restrict__ idx) {
    extern __shared__ unsigned long long sk[];  // the unit's keys
    __shared__ int hist[kSelectBins];
    __shared__ unsigned long long red[2][kSelectThreads / 32];
    __shared__ int wsum[2][kSelectThreads / 32];
    __shared__ int found[3];
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    constexpr int NW = kSelectThreads / 32;
    const long long unit = blockIdx.x;
    const int t = int(unit / P.H % P.T), b = int(unit / P.H / P.T);
    const AttendSeq seq = attend_seq(P, b, unit % ((long long)P.H * P.T) == 0 && tid == 0);
    const int lim = seq.tokens == 0 ? 0 : seq.len - (P.T - 1 - t);
    const int nb = (lim + (1 << P.block_shift) - 1) >> P.block_shift;
    int32_t* out = idx + unit * P.keep;
    if (nb <= P.keep) {
        for (int i = tid; i < P.keep; i += kSelectThreads) out[i] = i < nb ? i : -1;
        return;
    }
    // candidates: blocks [sink, nb - recent); nb > keep >= sink + recent
    const int c0 = sink, c1 = nb - recent;
    int need = P.keep - sink - recent;
    unsigned long long lo = ~0ull, hi = 0;
    for (int j = tid; j < nb; j += kSelectThreads) {
        const unsigned long long k = __ldg(keys + unit * blocks + j);
        sk[j] = k;
        if (j >= c0 && j < c1) {
            lo = min(lo, k);
            hi = max(hi, k);
        }
    }
    for (int o = 16; o; o >>= 1) {
        lo = min(lo, __shfl_xor_sync(~0u, lo, o));
        hi = max(hi, __shfl_xor_sync(~0u, hi, o));
    }
    if (lane == 0) {
        red[0][w] = lo;
        red[1][w] = hi;
    }
    __syncthreads();
    for (int i = 0; i < NW; ++i) {
        lo = min(lo, red[0][i]);
        hi = max(hi, red[1][i]);
    }
    // keys above hi are taken, keys below lo are not, `need` of those in between are still to be found
    unsigned long long border = 0;  // keys above it are taken, and of those equal to it ...
    int ties = 0;                   // ... this many, the lowest blocks first (-1: all)
    const bool none = need == 0;
    while (!none) {
        const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 11);
        for (int i = tid; i < kSelectBins; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        for (int j = c0 + tid; j < c1; j += kSelectThreads) {
            const unsigned long long k = sk[j];
            if (k >= lo && k <= hi) atomicAdd(&hist[int((k - lo) >> shift)], 1);
        }
        __syncthreads();
        // thread i holds bins from the top: [kSelectBins - 8 (i + 1), kSelectBins - 8 i)
        constexpr int PER = kSelectBins / kSelectThreads;
        const int top = kSelectBins - PER * (tid + 1);
        int mine = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) mine += hist[top + i];
        int inc = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(~0u, inc, o);
            if (lane >= o) inc += v;
        }
        if (lane == 31) wsum[0][w] = inc;
        __syncthreads();
        int before = inc - mine;
        for (int i = 0; i < w; ++i) before += wsum[0][i];
        if (before < need && before + mine >= need) {
            int at = before;
            for (int i = PER - 1; i >= 0; --i) {
                const int n = hist[top + i];
                if (at + n >= need) {
                    found[0] = top + i;
                    found[1] = need - at;
                    found[2] = n;
                    break;
                }
                at += n;
            }
        }
        __syncthreads();
        const unsigned long long new_lo = lo + ((unsigned long long)found[0] << shift);
        const unsigned long long width = shift == 0 ? 0 : (1ull << shift) - 1;
        const unsigned long long new_hi = hi - new_lo < width ? hi : new_lo + width;
        need = found[1];
        const int n = found[2];
        lo = new_lo;
        hi = new_hi;
        if (n == need || lo == hi) {  // the whole bin, or equal keys
            border = lo;
            ties = n == need ? -1 : need;
            break;
        }
        __syncthreads();
    }
    // ordered output: each thread a run of blocks, ranks by a scan
    const int per = (nb + kSelectThreads - 1) / kSelectThreads, j0 = min(nb, tid * per), j1 = min(nb, j0 + per);
    auto state = [&](int j) {  // 2: taken, 1: taken if among the first `ties` equal ones, 0: not
        if (j < c0 || j >= c1) return 2;
        if (none) return 0;
        const unsigned long long k = sk[j];
        if (ties < 0) return k >= border ? 2 : 0;
        return k > border ? 2 : k == border ? 1 : 0;
    };
    int nt = 0, ne = 0;
    for (int j = j0; j < j1; ++j) {
        const int s = state(j);
        nt += s == 2;
        ne += s == 1;
    }
    int it = nt, ie = ne;
    for (int o = 1; o < 32; o <<= 1) {
        const int a = __shfl_up_sync(~0u, it, o), e = __shfl_up_sync(~0u, ie, o);
        if (lane >= o) {
            it += a;
            ie += e;
        }
    }
    __syncthreads();
    if (lane == 31) {
        wsum[0][w] = it;
        wsum[1][w] = ie;
    }
    __syncthreads();
    int bt = it - nt, be = ie - ne;
    for (int i = 0; i < w; ++i) {
        bt += wsum[0][i];
        be += wsum[1][i];
    }
    for (int j = j0; j < j1; ++j) {
        const int s = state(j);
        if (s == 2 || (s == 1 && be < ties)) out[bt + min(be, max(ties, 0))] = j;
        bt += s == 2;
        be += s == 1;
    }
}

}  // namespace lagkv
