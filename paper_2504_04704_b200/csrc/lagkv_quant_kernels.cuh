// A cache in 8 bits with a scale for each block of rows and head: rows quantised as they are written, and read
// back -- sm_100a device code.
//
// Writing.  Block j of a (sequence, KV head) holds rows [jR, (j + 1) R).  With a = max |x| over the rows of the block that a
// call writes, and f the scale that they ask for,
//     int8:  f = a / 127 (correctly rounded),  code = x / s to the nearest whole number, ties to even,
//     e4m3:  f = the least power of two with a <= 448 f,  code = the nearest e4m3 to x / s,
// both at least 2^-126 (0 for a = 0),  s = f, or max(f, s before) where the block holds older rows, whose codes become code * (s before) / s, rounded
// again, when s grows.  A power of two costs e4m3 nothing (its steps are relative) and makes x / s and
// growing exact.  Codes are those of exact quotients (quant_factor).
//
// One read of the new rows: a group of threads fetches a block's new rows to shared memory (eight 16-byte pieces a thread, which
// nobody else reads, so that there is no barrier but the one of the reduction), two blocks ahead, finds the largest magnitude
// as integers (16-bit floats without their sign are ordered like them) and encodes.  Bound by HBM: 2 bytes read and 1
// written an element; 32 x 8 heads of 9728 rows of 128 channels in 316 us (int8) and 289 (e4m3) where the copy rate takes 292; kept rows by
// a list, 256 bytes at random places, 401 and 381.  (Registers only, 2-4 CTAs an SM: 610 and more.)
//
// Reading back: code * s in fp32, rounded to 16 bits; values that 16 bits do not hold become the largest that they do.
#pragma once
#include "lagkv_kernels.cuh"

namespace lagkv {

enum { FORM_INT8 = 0, FORM_E4M3 = 1 };

struct QuantParams {
    uint8_t* codes[2];                  // K, V
    float* scale[2];                    // [B, H, blocks]
    long long sb, sh, ss, page_stride;  // bytes
    const int32_t* block_table;
    long long num_pages, blocks;
    int B, H, D, S_cap, max_blocks, page_shift, block_shift;
    const int32_t* from_len;            // nullptr: 0
    const int32_t* seq_len;
    int32_t* status;
    // 16-bit rows: what is written, or where it is read back to; strides in elements
    uint16_t* rows[2];
    long long r_sb, r_sh, r_st;
    int T;                              // rows per (sequence, head) of it
    int at_positions;                   // position p is row p (else row p - from_len[b])
    const int32_t* take;                // [B, take_heads, n]: row of new row i; reading: position of row i
    int take_heads;
    int n;                              // rows a call may write per sequence; rows to read with `take`
    int per;                            // groups (writing) or CTAs (reading) per (sequence, head, tensor)
};

// Byte offset of row `r` of a head; -1: a page outside the pool (recorded).
__device__ __forceinline__ long long quant_offset(const QuantParams& P, int b, int h, int r) {
    if (P.block_table == nullptr) return (long long)b * P.sb + (long long)h * P.sh + (long long)r * P.ss;
    const int page = __ldg(P.block_table + (long long)b * P.max_blocks + (r >> P.page_shift));
    if (page < 0 || page >= P.num_pages) {
        record_status(P.status, ST_EINVAL, b);
        return -1;
    }
    return (long long)page * P.page_stride + (long long)h * P.sh + (long long)(r & ((1 << P.page_shift) - 1)) * P.ss;
}

template <int DT>
__device__ __forceinline__ void widen8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = Elem<DT>::lo(w[i]);
        x[2 * i + 1] = Elem<DT>::hi(w[i]);
    }
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// max of the magnitudes; the signs are anything, NaN stays
template <int DT>
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {
    uint32_t r;
    if (DT == 0)
        asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else
        asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return uint32_t(lo) | uint32_t(hi) << 16;
}

// The scale that a largest magnitude asks for.
template <int FORM>
__device__ __forceinline__ float quant_fit(float top) {
    if (top == 0.f) return 0.f;
    float f;
    if (FORM == FORM_INT8) {
        f = __fdiv_rn(top, 127.f);
    } else {
        // top = m 2^e, 1 <= m < 2 (a subnormal top: below the least scale all the same); 448 = 1.75 * 2^8
        const int bits = __float_as_int(top), e = (bits >> 23) - ((bits & 0x7fffff) <= 0x600000 ? 8 : 7);
        f = __int_as_float(max(e, 1) << 23);
    }
    return fmaxf(f, 0x1p-126f);
}

// a / b as an fp32 value that rounds to fewer bits as the exact quotient does: what fp32 does not hold is rounded to odd.
// a: up to 35 bits, b: 24; their 64-bit quotient is exact, or is as far from borders of fewer bits as the exact one.
__device__ __forceinline__ float odd_quotient(double a, float b) {
    const double q = a / b;
    const float f = __double2float_rz(q);
    return double(f) == q ? f : __int_as_float(__float_as_int(f) | 1);
}

// 1 / s; 0 for a scale of 0, and for one below 2^-126, which only another writer leaves and under which new rows are zeros: its
// inverse may be infinite, and 0 times that is no code.
__device__ __forceinline__ float quant_inverse(float s) { return s >= 0x1p-126f ? 1.f / s : 0.f; }

// Eight codes of x / s (e4m3: s a power of two).  int8: x * inv decides, see quant_factor(); with EXACT the remainder does.
template <int FORM, bool EXACT>
__device__ __forceinline__ uint2 quant_encode(const float (&x)[8], float s, float inv) {
    if (FORM == FORM_E4M3) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
        return make_uint2(pack_e4m3(y[0], y[1], y[2], y[3]), pack_e4m3(y[4], y[5], y[6], y[7]));
    }
    constexpr float kMagic = 12582912.f;  // 1.5 * 2^23: the sum's low byte is the whole number
    const f32x2 inv2 = pack2(inv, inv), magic2 = pack2(kMagic, kMagic);
    float n[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) unpack2(fma2(pack2(x[i], x[i + 1]), inv2, magic2), n[i], n[i + 1]);
    if (EXACT) {
        const float half = 0.5f * s;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float rest = fmaf(kMagic - n[i], s, x[i]);  // exact: x has at most 11 bits
            if (fabsf(rest) > half || (fabsf(rest) == half && (__float_as_int(n[i]) & 1))) n[i] += rest > 0.f ? 1.f : -1.f;
        }
    }
    auto low = [&](int i) { return uint32_t(__float_as_int(n[i])); };
    return make_uint2(__byte_perm(__byte_perm(low(0), low(1), 0x0040), __byte_perm(low(2), low(3), 0x0040), 0x5410),
                      __byte_perm(__byte_perm(low(4), low(5), 0x0040), __byte_perm(low(6), low(7), 0x0040), 0x5410));
}
// int8: the factor 1 / s, and whether it gives every value of the 16-bit type its code: only the value nearest to a border
// (n + 1/2) s, n < 127, can lie so near to it that the rounding of the factor matters, and each is tried.  Hardly a scale fails
// once the value at 63.5 (half the largest magnitude, which meets that border up to the rounding of s) has had its say in the last
// bit of the factor; the values of one that does are looked at one by one.  Warp-collective.
template <int DT>
__device__ __forceinline__ bool quant_factor(float s, int lane, float* inv) {
    float f = quant_inverse(s);
    auto wrong = [&](int n) {  // 0: the value nearest to the border above n gets its code, else which way it is off
        const float border = (float(n) + 0.5f) * s;
        uint32_t r;
        if (DT == 0)
            asm("cvt.rn.bf16x2.f32 %0, %1, %1;" : "=r"(r) : "f"(border));
        else
            asm("cvt.rn.f16x2.f32 %0, %1, %1;" : "=r"(r) : "f"(border));
        const float x = Elem<DT>::lo(r), above = fmaf(-float(n), s, x), half = 0.5f * s;  // exact where it is near half
        const bool up = above > half || (above == half && (n & 1));
        const bool taken = fmaf(x, f, 12582912.f) > 12582912.f + float(n);
        return x < INFINITY ? int(taken) - int(up) : 0;
    };
    const int off = wrong(63);
    f = __int_as_float(__float_as_int(f) - off);
    *inv = f;
    bool bad = false;
#pragma unroll
    for (int m = 0; m < 4; ++m) bad |= lane + 32 * m < 127 && wrong(lane + 32 * m) != 0;
    return !__any_sync(~0u, bad);
}

// Where 16 bytes of new row `i` of a call lie; nullptr: not in the source (recorded).
__device__ __forceinline__ const uint4* new_piece(const QuantParams& P, const uint16_t* src, const int32_t* take, int from, int i, int piece) {
    int row = P.at_positions ? from + i : i;
    if (take) row = __ldg(take + i);
    if (row >= 0 && row < P.T) return reinterpret_cast<const uint4*>(src + (long long)row * P.r_st) + piece;
    record_status(P.status, ST_EINVAL, -1);
    return nullptr;
}

// What hardly a call needs, out of the way of the registers of what every call does.
// The older codes of a block whose scale grows from `was` to `now`: rows of `to`, t of gt threads.
template <int FORM>
__device__ __noinline__ void quant_again(uint8_t* to, long long ss, int vpr, int rows, float was, float now, int t, int gt) {
    for (int i = t; i < rows * vpr * 4; i += gt) {
        uint32_t* p = reinterpret_cast<uint32_t*>(to + (long long)(i / (4 * vpr)) * ss) + i % (4 * vpr);
        const uint32_t w = *p;
        uint32_t y = 0;
        if (FORM == FORM_INT8) {
            for (int k = 0; k < 4; ++k) {  // 31 bits by 24: a 64-bit quotient rounds like the exact one
                const double q = rint(double(int8_t(w >> (8 * k))) * was / now);
                y |= (uint32_t(int(q)) & 255u) << (8 * k);
            }
        } else {
            uint32_t x[2];
            Elem<2>::expand(w, x);
            const double f = was;  // codes of 4 bits, scales of 24
            y = pack_e4m3(odd_quotient(Elem<1>::lo(x[0]) * f, now), odd_quotient(Elem<1>::hi(x[0]) * f, now),
                          odd_quotient(Elem<1>::lo(x[1]) * f, now), odd_quotient(Elem<1>::hi(x[1]) * f, now));
        }
        *p = y;
    }
}
// New rows [i0, i1) of a call with values that are not finite, or under an e4m3 scale that is no power of two: read again.
template <int DT, int FORM>
__device__ __noinline__ void quant_with_care(const QuantParams& P, const uint16_t* src, const int32_t* take, int from, int i0, int i1,
                                             uint8_t* to, float s, int t, int gt) {
    const int cpr = P.D / 8;
    const double limit = double(s) * (FORM == FORM_INT8 ? 127.0 : 448.0);
    for (int c = t; c < (i1 - i0) * cpr; c += gt) {
        const int r = c / cpr, piece = c % cpr;
        const uint4* p = new_piece(P, src, take, from, i0 + r, piece);
        const uint4 v = p ? __ldg(p) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint8_t* out = to + (long long)r * P.ss + piece * 8;
        for (int i = 0; i < 8; ++i) {
            const float x = i & 1 ? Elem<DT>::hi(w[i >> 1]) : Elem<DT>::lo(w[i >> 1]);
            const double y = x != x || s == 0.f ? 0.0 : fmin(fmax(double(x), -limit), limit);
            const float by = s == 0.f ? 1.f : s;
            out[i] = FORM == FORM_INT8 ? uint8_t(int(rint(y / by))) : uint8_t(pack_e4m3(odd_quotient(y, by), 0.f, 0.f, 0.f));
        }
    }
}

constexpr int kQuantPieces = 8, kQuantStages = 3;  // 16-byte pieces of new rows of a thread and block, blocks in flight
template <int GT>
struct QuantWriteGeo {
    static constexpr int NT = GT > 256 ? GT : 256, GROUPS = NT / GT;
    static constexpr int STAGE = NT * kQuantPieces * 16, SMEM = kQuantStages * STAGE;
};

// GT threads take a block's new rows, at most 8 times the GT / (D / 8) rows that they fetch a piece each of.
template <int DT, int FORM, int GT>
__global__ void __launch_bounds__(QuantWriteGeo<GT>::NT, GT > 256 ? 1 : 2)
lagkv_quant_write_kernel(const __grid_constant__ QuantParams P) {
    using G = QuantWriteGeo<GT>;
    constexpr uint32_t kInf = DT == 0 ? 0x7f80u : 0x7c00u;
    extern __shared__ __align__(128) uint4 ring[];
    __shared__ uint32_t tops[2][G::NT / 32];
    const int tid = threadIdx.x, t = tid % GT, group = tid / GT;
    const uint32_t id = blockIdx.x * G::GROUPS + group, unit = id / uint32_t(P.per);
    if (unit >= 2u * P.B * P.H) return;  // a whole group: its barriers are its own
    const int slot = int(id % uint32_t(P.per)), which = int(unit & 1), h = int((unit >> 1) % P.H), b = int((unit >> 1) / P.H);
    const int from = P.from_len ? __ldg(P.from_len + b) : 0, seq = __ldg(P.seq_len + b);
    if (from < 0 || seq < from || seq > P.S_cap || seq - from > P.n || (P.take == nullptr && P.at_positions && seq > P.T)) {
        if (t == 0) record_status(P.status, ST_EINVAL, b);
        return;
    }
    // a thread keeps its piece of a row and goes on by `pass` rows (D = 96: some threads have none)
    const int cpr = P.D / 8, pass = GT / cpr, r0 = t / cpr, piece = t - r0 * cpr;
    const int first = from >> P.block_shift, blocks = seq > from ? (seq + (1 << P.block_shift) - 1) >> P.block_shift : 0;
    const uint16_t* src = P.rows[which] + (long long)b * P.r_sb + (long long)h * P.r_sh;
    const int32_t* take = P.take ? P.take + ((long long)b * P.take_heads + (P.take_heads > 1 ? h : 0)) * P.n : nullptr;
    uint8_t* codes = P.codes[which];
    float* scales = P.scale[which] + ((long long)b * P.H + h) * P.blocks;
    auto place = [&](int stage, int k) { return ring + (stage * kQuantPieces + k) * G::NT + tid; };
    int row[kQuantPieces];  // take: rows of the source for the block that is fetched next, looked up a block ahead and not looked at before
    auto look = [&](int j) {
        if (take == nullptr) return;
        const int i0 = max(from, j << P.block_shift) + r0 - from, e = j < blocks ? min(seq, (j + 1) << P.block_shift) - from : 0;
#pragma unroll
        for (int k = 0; k < kQuantPieces; ++k) row[k] = r0 < pass && i0 + k * pass < e ? __ldg(take + i0 + k * pass) : 0;
    };
    auto fetch = [&](int j, int stage) {
        if (j < blocks) {
            const int i0 = max(from, j << P.block_shift) + r0, e = min(seq, (j + 1) << P.block_shift);
            const uint16_t* p = src + (long long)(P.at_positions ? i0 : i0 - from) * P.r_st + piece * 8;
#pragma unroll
            for (int k = 0; k < kQuantPieces; ++k) {
                bool ok = r0 < pass && i0 + k * pass < e;  // what is not there becomes zeros
                if (take) {
                    const bool in = row[k] >= 0 && row[k] < P.T;
                    if (ok && !in) record_status(P.status, ST_EINVAL, b);
                    ok = ok && in;
                    p = src + (long long)row[k] * P.r_st + piece * 8;
                }
                asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(smem_u32(place(stage, k))), "l"(ok ? p : src), "r"(ok ? 16 : 0)
                             : "memory");
                if (!take) p += pass * P.r_st;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        look(j + P.per);
    };
    int turn = 0;
    auto largest = [&](uint32_t top) {  // of a group's packed magnitudes
#pragma unroll
        for (int o = 16; o; o >>= 1) top = max_u16x2(top, __shfl_xor_sync(~0u, top, o));
        if (GT > 32) {
            if ((tid & 31) == 0) tops[turn][tid >> 5] = top;
            asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(GT) : "memory");
#pragma unroll
            for (int k = 0; k < GT / 32; ++k) top = max_u16x2(top, tops[turn][group * (GT / 32) + k]);
            turn ^= 1;  // written again two barriers on, when all have read
        }
        return max(top & 0xffffu, top >> 16);
    };
    int stage = 0;
    look(first + slot);
#pragma unroll 1
    for (int i = 0; i < kQuantStages - 1; ++i) fetch(first + slot + i * P.per, i);
    for (int j = first + slot; j < blocks; j += P.per) {
        fetch(j + (kQuantStages - 1) * P.per, stage == 0 ? kQuantStages - 1 : stage - 1);
        const int start = j << P.block_shift, a = max(from, start), e = min(seq, start + (1 << P.block_shift));
        const long long off = quant_offset(P, b, h, start);
        const bool older = start < from;
        const float was = older ? scales[j] : 0.f;
        asm volatile("cp.async.wait_group %0;" ::"n"(kQuantStages - 1) : "memory");
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < kQuantPieces; ++k) {
            const uint4 v = *place(stage, k);
            top = max_abs2<DT>(top, max_abs2<DT>(max_abs2<DT>(v.x, v.y), max_abs2<DT>(v.z, v.w)));
        }
        uint32_t high = largest(top & 0x7fff7fffu);
        const bool odd = high >= kInf;
        if (odd) {  // values that are not finite: recorded, and they do not count
            if (t == 0) record_status(P.status, ST_EINVAL, b);
            top = 0;
#pragma unroll 1
            for (int k = 0; k < kQuantPieces; ++k) {
                const uint4 v = *place(stage, k);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if ((w[i] & 0x7fffu) < kInf) top = max(top, w[i] & 0x7fffu);
                    if ((w[i] >> 16 & 0x7fffu) < kInf) top = max(top, w[i] >> 16 & 0x7fffu);
                }
            }
            high = largest(top);
        }
        const float s = fmaxf(quant_fit<FORM>(Elem<DT>::lo(high)), was);
        if (off >= 0) {  // else: no page
            uint8_t* to = codes + off;
            if (t == 0 && !(older && s == was)) scales[j] = s;  // every thread has read it: largest() lies between
            if (odd || (FORM == FORM_E4M3 && (__float_as_int(s) & 0x7fffff))) {
                quant_with_care<DT, FORM>(P, src, take, from, a - from, e - from, to + (long long)(a - start) * P.ss, s, t, GT);
            } else {
                float inv = quant_inverse(s);
                const bool plain = FORM == FORM_E4M3 || quant_factor<DT>(s, tid & 31, &inv);
                const int mine = r0 < pass ? (e - a - r0 + pass - 1) / pass : 0;  // pieces of this thread, if positive
                uint8_t* out = to + (long long)(a - start + r0) * P.ss + piece * 8;
                if (!plain) {
#pragma unroll 1
                    for (int k = 0; k < min(mine, kQuantPieces); ++k) {
                        float x[8];
                        widen8<DT>(*place(stage, k), x);
                        *reinterpret_cast<uint2*>(out) = quant_encode<FORM, true>(x, s, inv);
                        out += pass * P.ss;
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < kQuantPieces; ++k) {
                        if (k < mine) {
                            float x[8];
                            widen8<DT>(*place(stage, k), x);
                            *reinterpret_cast<uint2*>(out) = quant_encode<FORM, false>(x, s, inv);
                        }
                        out += pass * P.ss;
                    }
                }
            }
            if (older && s > was) quant_again<FORM>(to, P.ss, P.D / 16, a - start, was, s, t, GT);
        }
        if (++stage == kQuantStages) stage = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// Eight codes times their scale, in 16 bits.
template <int DT, int FORM>
__device__ __forceinline__ uint4 quant_decode(const uint2& v, float s) {
    constexpr float kMost = DT == 0 ? 0x1.fep127f : 65504.f;
    const bool wide = s > kMost / 512.f;  // only then a code may stand for more
    const uint32_t w[2] = {v.x, v.y};
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float x[4];
        if (FORM == FORM_INT8) {  // 2^23 + 128 + code
            const uint32_t u = w[i] ^ 0x80808080u;
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540 + k)) - 8388736.f;
        } else {
            uint32_t p[2];
            Elem<2>::expand(w[i], p);
            x[0] = Elem<1>::lo(p[0]);
            x[1] = Elem<1>::hi(p[0]);
            x[2] = Elem<1>::lo(p[1]);
            x[3] = Elem<1>::hi(p[1]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] *= s;
        if (wide) {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = x[k] != x[k] ? x[k] : fminf(fmaxf(x[k], -kMost), kMost);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (DT == 0)
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y[2 * i + k]) : "f"(x[2 * k + 1]), "f"(x[2 * k]));
            else
                asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y[2 * i + k]) : "f"(x[2 * k + 1]), "f"(x[2 * k]));
        }
    }
    return make_uint4(y[0], y[1], y[2], y[3]);
}

constexpr int kReadThreads = 256, kReadPieces = 4;  // 8-code pieces of a thread that are in flight

// CTAs walk the rows of a (sequence, head, tensor) in strides.  Without `take` position p goes to row p of the output; with
// it position take[i] goes to row i.  A thread takes eight codes at a time, so that a warp's stores lie side by side.
// 32 x 8 heads of 4864 to 9728 e4m3 rows of 128 channels: 236 us, HBM at 95 % of the copy rate (16 codes a thread, whose two
// stores leave gaps: 272; a persistent grid with equal shares of all rows 271 and more, the next rows' loads ahead of the stores
// 327: what counts is how many warps there are).
template <int DT, int FORM>
__global__ void __launch_bounds__(kReadThreads)
lagkv_quant_read_kernel(const __grid_constant__ QuantParams P) {
    const int unit = blockIdx.x / P.per, slot = blockIdx.x % P.per, which = unit & 1, h = (unit >> 1) % P.H, b = (unit >> 1) / P.H;
    if (P.rows[which] == nullptr) return;
    const int from = P.from_len ? __ldg(P.from_len + b) : 0, seq = __ldg(P.seq_len + b);
    if (from < 0 || seq < from || seq > P.S_cap || (P.take == nullptr && seq > P.T)) {
        if (threadIdx.x == 0) record_status(P.status, ST_EINVAL, b);
        return;
    }
    // a thread keeps its piece of a row and goes on by `pass` rows (D = 96: some threads have none)
    const int cpr = P.D / 8, pass = kReadThreads / cpr, r0 = int(threadIdx.x) / cpr, piece = int(threadIdx.x) - r0 * cpr;
    const int32_t* take = P.take ? P.take + ((long long)b * P.H + h) * P.n : nullptr;
    const int begin = take ? 0 : from, end = take ? P.n : seq;
    uint16_t* out = P.rows[which] + (long long)b * P.r_sb + (long long)h * P.r_sh + piece * 8;
    const uint8_t* codes = P.codes[which] + piece * 8;
    const float* scales = P.scale[which] + ((long long)b * P.H + h) * P.blocks;
    if (r0 >= pass) return;
    for (long long i0 = begin + (long long)slot * pass * kReadPieces + r0; i0 < end; i0 += (long long)P.per * pass * kReadPieces) {
        uint2 v[kReadPieces];
        float s[kReadPieces];
        uint32_t there = 0;
#pragma unroll
        for (int k = 0; k < kReadPieces; ++k) {
            const long long i = i0 + k * pass;
            if (i >= end) continue;
            const int p = take ? __ldg(take + i) : int(i);
            if (take && (p < 0 || p >= seq)) {
                record_status(P.status, ST_EINVAL, b);
                continue;
            }
            const long long off = quant_offset(P, b, h, p);
            if (off < 0) continue;
            there |= 1u << k;
            v[k] = __ldcs(reinterpret_cast<const uint2*>(codes + off));
            s[k] = scales[p >> P.block_shift];
        }
#pragma unroll
        for (int k = 0; k < kReadPieces; ++k)
            if (there >> k & 1) __stcs(reinterpret_cast<uint4*>(out + (i0 + k * pass) * P.r_st), quant_decode<DT, FORM>(v[k], s[k]));
    }
}

}  // namespace lagkv
