// A cache in 8 bits with a scale for each block of rows and head: rows quantised as they are written, and read
// back -- sm_100a device code.
//
// Writing.  Block j of a (sequence, KV head) holds rows [jR, (j + 1) R).  With a = max |x| over the rows of the block that a
// call writes, and f the scale that they ask for,
//     int8:  f = a / 127 (correctly rounded),  code = x / s to the nearest whole number, ties to even,
//     e4m3:  f = the least power of two with a <= 448 f,  code = the nearest e4m3 to x / s,
// both at least 2^-126 (0 for a = 0),  s = f, or max(f, s before) where the block holds older rows, whose codes become code * (s before) / s, rounded
// again, when s grows.  A power of two costs e4m3 nothing (its steps are relative) and makes x / s and
// growing exact.  Codes are those of exact quotients: int8 looks at quotients next to a border again, with the remainder that
// an fma gives exactly.
//
// One read of the new rows: a group of threads holds a block's new rows in registers (eight 16-byte pieces a thread),
// finds the largest magnitude as integers (16-bit floats without their sign are ordered like them) and encodes from
// the registers.  Bound by HBM: 2 bytes read and 1 written an element.
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
    uint32_t by_cpr;                    // ceil(65536 / 16-bit pieces of a row)
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

// Eight codes of x / s.
template <int FORM>
__device__ __forceinline__ uint2 quant_encode(const float (&x)[8], float s, float inv) {
    if (FORM == FORM_E4M3) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
        if (__float_as_int(s) & 0x7fffff) {  // no power of two: not a scale from here
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = odd_quotient(x[i], s);
        }
        return make_uint2(pack_e4m3(y[0], y[1], y[2], y[3]), pack_e4m3(y[4], y[5], y[6], y[7]));
    }
    constexpr float kMagic = 12582912.f;  // 1.5 * 2^23: the sum's low byte is the whole number
    float n[8], far = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = x[i] * inv;
        n[i] = q + kMagic;
        far = fmaxf(far, fabsf(q - (n[i] - kMagic)));
    }
    if (far > 0.4999f) {  // q is off by at most 127.5 * 1.5 * 2^-23: next to a border the remainder decides
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float whole = n[i] - kMagic, rest = fmaf(-whole, s, x[i]), half = 0.5f * s;
            const bool odd = __float_as_int(n[i]) & 1;
            if (fabsf(rest) > half || (fabsf(rest) == half && odd)) n[i] += rest > 0.f ? 1.f : -1.f;
        }
    }
    auto low = [&](int i) { return uint32_t(__float_as_int(n[i])); };
    return make_uint2(__byte_perm(__byte_perm(low(0), low(1), 0x0040), __byte_perm(low(2), low(3), 0x0040), 0x5410),
                      __byte_perm(__byte_perm(low(4), low(5), 0x0040), __byte_perm(low(6), low(7), 0x0040), 0x5410));
}

// 16 codes whose scale grows from `was` to `now`.
template <int FORM>
__device__ __forceinline__ uint4 quant_again(const uint4& v, float was, float now) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t y[4];
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
        if (FORM == FORM_INT8) {
            y[i] = 0;
            for (int k = 0; k < 4; ++k) {  // 31 bits by 24: a 64-bit quotient rounds like the exact one
                const double q = rint(double(int8_t(w[i] >> (8 * k))) * was / now);
                y[i] |= (uint32_t(int(q)) & 255u) << (8 * k);
            }
        } else {
            uint32_t p[2];
            Elem<2>::expand(w[i], p);
            const double f = was;  // codes of 4 bits, scales of 24
            y[i] = pack_e4m3(odd_quotient(Elem<1>::lo(p[0]) * f, now), odd_quotient(Elem<1>::hi(p[0]) * f, now),
                             odd_quotient(Elem<1>::lo(p[1]) * f, now), odd_quotient(Elem<1>::hi(p[1]) * f, now));
        }
    }
    return make_uint4(y[0], y[1], y[2], y[3]);
}

constexpr int kQuantPieces = 8;  // 16-byte pieces of new rows that a thread holds

// GT threads take a block's new rows: at least an eighth of their 16-byte pieces.
template <int DT, int FORM, int GT>
__global__ void __launch_bounds__(GT > 256 ? GT : 256)
lagkv_quant_write_kernel(const __grid_constant__ QuantParams P) {
    constexpr int NT = GT > 256 ? GT : 256, GROUPS = NT / GT;
    constexpr uint32_t kInf = DT == 0 ? 0x7f80u : 0x7c00u;
    __shared__ uint32_t tops[2][NT / 32];
    const int tid = threadIdx.x, t = tid % GT, group = tid / GT;
    const long long unit = ((long long)blockIdx.x * GROUPS + group) / P.per;
    if (unit >= 2ll * P.B * P.H) return;  // a whole group: its barriers are its own
    const int slot = int(((long long)blockIdx.x * GROUPS + group) % P.per);
    const int which = int(unit & 1), h = int((unit >> 1) % P.H), b = int((unit >> 1) / P.H);
    const int from = P.from_len ? __ldg(P.from_len + b) : 0, seq = __ldg(P.seq_len + b);
    if (from < 0 || seq < from || seq > P.S_cap || seq - from > P.n || (P.take == nullptr && P.at_positions && seq > P.T)) {
        if (t == 0) record_status(P.status, ST_EINVAL, b);
        return;
    }
    const int cpr = P.D / 8, first = from >> P.block_shift, blocks = (seq + (1 << P.block_shift) - 1) >> P.block_shift;
    const uint16_t* src = P.rows[which] + (long long)b * P.r_sb + (long long)h * P.r_sh;
    const int32_t* take = P.take ? P.take + ((long long)b * P.take_heads + (P.take_heads > 1 ? h : 0)) * P.n : nullptr;
    uint8_t* codes = P.codes[which];
    float* scales = P.scale[which] + ((long long)b * P.H + h) * P.blocks;
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
    for (int j = first + slot; j < blocks && seq > from; j += P.per) {
        const int start = j << P.block_shift, a = max(from, start), e = min(seq, start + (1 << P.block_shift));
        const long long off = quant_offset(P, b, h, start);
        const bool older = start < from;
        const float was = older ? scales[j] : 0.f;
        uint4 v[kQuantPieces];
#pragma unroll
        for (int k = 0; k < kQuantPieces; ++k) {
            const int c = k * GT + t, r = int(uint32_t(c) * P.by_cpr >> 16);
            v[k] = make_uint4(0u, 0u, 0u, 0u);
            if (a + r < e) {
                int from_row = P.at_positions ? a + r : a + r - from;
                if (take) from_row = __ldg(take + (a + r - from));
                if (from_row >= 0 && from_row < P.T)
                    v[k] = __ldg(reinterpret_cast<const uint4*>(src + (long long)from_row * P.r_st) + (c - r * cpr));
                else
                    record_status(P.status, ST_EINVAL, b);
            }
        }
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < kQuantPieces; ++k)
            top = max_u16x2(top, max_u16x2(max_u16x2(v[k].x & 0x7fff7fffu, v[k].y & 0x7fff7fffu), max_u16x2(v[k].z & 0x7fff7fffu, v[k].w & 0x7fff7fffu)));
        uint32_t high = largest(top);
        const bool odd = high >= kInf;
        if (odd) {  // values that are not finite do not count: recorded, NaN becomes 0, infinities the largest code
            if (t == 0) record_status(P.status, ST_EINVAL, b);
            top = 0;
            auto clean = [&](uint32_t& w) {
                if ((w & 0x7fffu) > kInf) w &= 0xffff0000u;
                if ((w >> 16 & 0x7fffu) > kInf) w &= 0x0000ffffu;
                if ((w & 0x7fffu) < kInf) top = max(top, w & 0x7fffu);
                if ((w >> 16 & 0x7fffu) < kInf) top = max(top, w >> 16 & 0x7fffu);
            };
#pragma unroll
            for (int k = 0; k < kQuantPieces; ++k) {
                clean(v[k].x);
                clean(v[k].y);
                clean(v[k].z);
                clean(v[k].w);
            }
            high = largest(top);
        }
        const float fit = quant_fit<FORM>(Elem<DT>::lo(high)), s = fmaxf(fit, was);
        const float inv = s > 0.f ? 1.f / s : 0.f, limit = (FORM == FORM_INT8 ? 127.f : 448.f) * s;
        if (off < 0) continue;  // no page
        uint8_t* to = codes + off;
        if (older && s > was && was > 0.f) {
            const int vpr = P.D / 16, n = (a - start) * vpr;
            for (int i = t; i < n; i += GT) {
                uint4* p = reinterpret_cast<uint4*>(to + (long long)(i / vpr) * P.ss) + i % vpr;
                *p = quant_again<FORM>(*p, was, s);
            }
        }
        if (t == 0 && !(older && s == was)) scales[j] = s;  // every thread has read it: largest() lies between
#pragma unroll
        for (int k = 0; k < kQuantPieces; ++k) {
            const int c = k * GT + t, r = int(uint32_t(c) * P.by_cpr >> 16);
            if (a + r < e) {
                float x[8];
                widen8<DT>(v[k], x);
                if (odd) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = fminf(fmaxf(x[i], -limit), limit);
                    if (s == 0.f) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = 0.f;
                    }
                }
                *reinterpret_cast<uint2*>(to + (long long)(a - start + r) * P.ss + (c - r * cpr) * 8) = quant_encode<FORM>(x, s, inv);
            }
        }
    }
}

// 16 codes times their scale, in 16 bits.
template <int DT, int FORM>
__device__ __forceinline__ void quant_decode(const uint4& v, float s, uint4 (&out)[2]) {
    constexpr float kMost = DT == 0 ? 0x1.fep127f : 65504.f;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
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
        for (int k = 0; k < 4; ++k) {
            const float z = x[k] * s;
            x[k] = z != z ? z : fminf(fmaxf(z, -kMost), kMost);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (DT == 0)
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y[2 * i + k]) : "f"(x[2 * k + 1]), "f"(x[2 * k]));
            else
                asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y[2 * i + k]) : "f"(x[2 * k + 1]), "f"(x[2 * k]));
        }
    }
    out[0] = make_uint4(y[0], y[1], y[2], y[3]);
    out[1] = make_uint4(y[4], y[5], y[6], y[7]);
}

constexpr int kReadThreads = 256, kReadPieces = 4;  // 16-code pieces of a thread that are in flight

// CTAs walk the rows of a (sequence, head, tensor) in strides.  Without `take` position p goes to row p of the output; with
// it position take[i] goes to row i.
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
    const int vpr = P.D / 16, first = P.take ? 0 : from, n = P.take ? P.n : seq - from;
    const int32_t* take = P.take ? P.take + ((long long)b * P.H + h) * P.n : nullptr;
    uint16_t* out = P.rows[which] + (long long)b * P.r_sb + (long long)h * P.r_sh;
    const uint8_t* codes = P.codes[which];
    const float* scales = P.scale[which] + ((long long)b * P.H + h) * P.blocks;
    const long long total = (long long)n * vpr, step = (long long)P.per * kReadThreads * kReadPieces;
    for (long long i0 = (long long)slot * kReadThreads * kReadPieces + threadIdx.x; i0 < total; i0 += step) {
        uint4 v[kReadPieces];
        float s[kReadPieces];
        int row[kReadPieces];
#pragma unroll
        for (int k = 0; k < kReadPieces; ++k) {
            const long long i = i0 + k * kReadThreads;
            row[k] = -1;
            if (i >= total) continue;
            const int r = int((i >> 32) == 0 ? uint32_t(i) / uint32_t(vpr) : i / vpr), p = take ? __ldg(take + r) : first + r;
            if (take && (p < 0 || p >= seq)) {
                record_status(P.status, ST_EINVAL, b);
                continue;
            }
            const long long off = quant_offset(P, b, h, p);
            if (off < 0) continue;
            row[k] = first + r;
            v[k] = __ldcs(reinterpret_cast<const uint4*>(codes + off) + (i - (long long)r * vpr));
            s[k] = scales[p >> P.block_shift];
        }
#pragma unroll
        for (int k = 0; k < kReadPieces; ++k) {
            if (row[k] < 0) continue;
            const long long i = i0 + k * kReadThreads;
            uint4 y[2];
            quant_decode<DT, FORM>(v[k], s[k], y);
            uint4* to = reinterpret_cast<uint4*>(out + (long long)row[k] * P.r_st) + 2 * (i - (long long)(row[k] - first) * vpr);
            __stcs(to, y[0]);
            __stcs(to + 1, y[1]);
        }
    }
}

}  // namespace lagkv
