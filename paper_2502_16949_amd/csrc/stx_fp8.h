// 8-bit floats and typed row access, shared by stx_norm.hip, stx_q8.hip, stx_q8_matmul.hip and stx_adamw.hip.
//
// Work on 8-bit blocks is laid out by "octets": 16 consecutive lanes (a row of the data-parallel moves) own the 128 elements of
// a block, 8 each, so that a block's largest magnitude is four moves inside that row.  Octets of 16-bit elements are 8
// consecutive ones (one 16-byte access); those of fp32 are two quads 64 elements apart, so that each of the two 16-byte
// accesses of a lane row is contiguous.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "stx.h"

namespace stx {

constexpr int kBlock = 128;            // elements that share a scale

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// Vectors at the alignment of their elements: the hardware takes any multiple of an element.
typedef float f4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x8u_t __attribute__((ext_vector_type(8), aligned(2)));
typedef uint32_t u32x4u_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32u_t __attribute__((aligned(1)));

template <class T> __device__ inline float to_float(uint16_t bits);
template <> __device__ inline float to_float<bf16_t>(uint16_t bits) { return __builtin_bit_cast(float, (uint32_t)bits << 16); }
template <> __device__ inline float to_float<f16_t>(uint16_t bits) { return (float)__builtin_bit_cast(f16_t, bits); }
// rounded to nearest even
template <class T> __device__ inline uint16_t from_float(float v) { return __builtin_bit_cast(uint16_t, (T)v); }

// Position of element j of the octet that lane `l16` of block `blk` owns.
template <class T>
__device__ inline int octet_pos(int blk, int l16, int j)
{
    return sizeof(T) == 4 ? blk * kBlock + (j >> 2) * 64 + 4 * l16 + (j & 3) : blk * kBlock + 8 * l16 + j;
}

// An octet as it lies in memory.  Requesting one and making floats of it are two functions, and a kernel requests all that it needs
// first.  Nothing in a request depends on the row's end but its address: an access that would reach behind the end is moved back to
// end there, and its elements are shifted into place when they are made floats, by wavefronts that hold such a one (a branch around
// the request would make the kernel wait for it at the branch's end).
template <class T> struct Octet { uint32_t w[sizeof(T) * 2]; };

// The octet that lane l16 of block blk owns of a row of n elements (n >= 0).
template <class T>
__device__ inline Octet<T> request_octet(const T *row, int blk, int l16, int64_t n)
{
    Octet<T> o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = (int64_t)blk * kBlock + h * 64 + 4 * l16;
            f4u_t q = {0.f, 0.f, 0.f, 0.f};
            if (n >= 4) {
                q = *reinterpret_cast<const f4u_t *>(row + min(at, n - 4));
            } else {
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (at + j < n) q[j] = row[at + j];
                __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0) here, and not in front of the other branch's request
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float f = q[j];      // (a bit cast of a vector's element itself takes the first one)
                o.w[4 * h + j] = __builtin_bit_cast(uint32_t, f);
            }
        }
    } else {
        const uint16_t *r16 = reinterpret_cast<const uint16_t *>(row);
        const int64_t at = (int64_t)blk * kBlock + 8 * l16;
        u32x4u_t q = {0u, 0u, 0u, 0u};
        if (n >= 8) {
            q = *reinterpret_cast<const u32x4u_t *>(r16 + min(at, n - 8));
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (at + j < n) q[j / 2] |= (uint32_t)r16[at + j] << (16 * (j & 1));
            __builtin_amdgcn_s_waitcnt(0x0f70);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) o.w[j] = q[j];
    }
    return o;
}
// Puts the elements of request_octet(row, blk, l16, n) into place; 0 behind the row's end.
template <class T>
__device__ inline void settle_octet(Octet<T> &o, int blk, int l16, int64_t n)
{
    constexpr int N = 16 / sizeof(T);      // elements of an access
    if (n < N || !__ballot(octet_pos<T>(blk, l16, 8 - N) + N > n)) return;
#pragma unroll
    for (int h = 0; h < 8 / N; ++h) {
        const int64_t over = octet_pos<T>(blk, l16, h * N) + N - n;
        const int by = (int)(over < 0 ? 0 : over > N ? N : over);
        uint32_t *w = o.w + 4 * h;
#pragma unroll
        for (int u = 4; u >= 1; u >>= 1)   // whole words down
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = (by * (int)sizeof(T) / 4 & u) ? (j + u < 4 ? w[j + u] : 0u) : w[j];
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = (by & 1) ? w[j] >> 16 | (j < 3 ? w[j + 1] << 16 : 0u) : w[j];
        }
    }
}
// The elements of request_octet(row, blk, l16, n) as floats; 0 behind the row's end.
template <class T>
__device__ inline void octet_floats(Octet<T> o, int blk, int l16, int64_t n, float (&v)[8])
{
    settle_octet(o, blk, l16, n);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (sizeof(T) == 4) v[j] = __builtin_bit_cast(float, o.w[j]);
        else v[j] = to_float<T>((uint16_t)(o.w[j / 2] >> (16 * (j & 1))));
    }
}

// Of a row of floats, in the octets of T: a weight goes with the rows that it scales.
template <class T>
__device__ inline void load_octet_as(const float *row, int blk, int l16, int64_t n, float (&v)[8])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t at = octet_pos<T>(blk, l16, 4 * h);
        if (at + 4 <= n) {
            const f4u_t q = *reinterpret_cast<const f4u_t *>(row + at);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * h + j] = q[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * h + j] = at + j < n ? row[at + j] : 0.f;
        }
    }
}

// A store past the caches, if `past`.  (Without something between them the compiler makes one plain store of the two.)
#define STX_STORE_PAST(TYPE)                                       \
    __device__ inline void store_past(TYPE v, TYPE *at, bool past) \
    {                                                            \
        if (past) {                                              \
            asm volatile("");                                    \
            __builtin_nontemporal_store(v, at);                  \
            asm volatile("");                                    \
        } else {                                                 \
            *at = v;                                             \
        }                                                        \
    }
STX_STORE_PAST(f4u_t)
STX_STORE_PAST(u16x8u_t)
#undef STX_STORE_PAST

// Rounds v to T and, if row is not null, stores it there; past the caches, if `past`.
template <class T>
__device__ inline void round_store_octet(T *row, int blk, int l16, int64_t n, float (&v)[8], bool past)
{
    if constexpr (sizeof(T) == 4) {
        if (!row) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = (int64_t)blk * kBlock + h * 64 + 4 * l16;
            if (at + 4 <= n) {
                const f4u_t q = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                store_past(q, reinterpret_cast<f4u_t *>(row + at), past);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (at + j < n) row[at + j] = v[4 * h + j];
            }
        }
    } else {
        u16x8u_t q;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            q[j] = from_float<T>(v[j]);
            v[j] = to_float<T>(q[j]);
        }
        if (!row) return;
        uint16_t *r16 = reinterpret_cast<uint16_t *>(row);
        const int64_t at = (int64_t)blk * kBlock + 8 * l16;
        if (at + 8 <= n) {
            store_past(q, reinterpret_cast<u16x8u_t *>(r16 + at), past);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at + j < n) r16[at + j] = q[j];
        }
    }
}

// Largest of one value per lane over the 16 lanes of its row; every lane receives it.
__device__ inline uint32_t row16_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));   // rotated by 8, 4, 2, 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));
    return v;
}

constexpr uint32_t kInfBits = 0x7f800000u;
__device__ inline uint32_t abs_bits(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
__device__ inline uint32_t finite_bits(float v) { const uint32_t b = abs_bits(v); return b < kInfBits ? b : 0u; }

// Largest finite magnitudes, as bits of an fp32: over N numbers, and over N pairs of 16-bit numbers, of each half.  What is not
// finite is left out in a second pass, by wavefronts that have met one.
template <int N>
__device__ inline uint32_t largest(const float *v)
{
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) m = max(m, abs_bits(v[j]));
    if (__ballot(m >= kInfBits)) {
        m = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) m = max(m, finite_bits(v[j]));
    }
    return m;
}
template <class T, int N>
__device__ inline void largest_pair(const uint32_t *w, uint32_t &lo, uint32_t &hi)
{
    typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
    constexpr uint32_t inf = __is_same(T, bf16_t) ? 0x7f80u : 0x7c00u;
    u16x2_t m = {0, 0};
#pragma unroll
    for (int j = 0; j < N; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, w[j] & 0x7fff7fffu));
    lo = m.x;
    hi = m.y;
    if (__ballot(max(lo, hi) >= inf)) {
        lo = hi = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t a = w[j] & 0x7fffu, b = w[j] >> 16 & 0x7fffu;
            lo = max(lo, a < inf ? a : 0u);
            hi = max(hi, b < inf ? b : 0u);
        }
    }
    lo = __builtin_bit_cast(uint32_t, to_float<T>((uint16_t)lo));
    hi = __builtin_bit_cast(uint32_t, to_float<T>((uint16_t)hi));
}
template <class T>
__device__ inline uint32_t largest(const Octet<T> &o)
{
    if constexpr (sizeof(T) == 4) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(float, o.w[j]);
        return largest<8>(v);
    } else {
        uint32_t lo, hi;
        largest_pair<T, 4>(o.w, lo, hi);
        return max(lo, hi);
    }
}

// The exponent byte of a block's scale from the bits of its largest finite magnitude: both formats' largest numbers are 1.75
// times a power of two, so a magnitude 1.f 2^E needs 2^(E - 8), or one power more where 1.f > 1.75.
template <int FORMAT>
__device__ inline uint32_t block_scale(uint32_t most)
{
    constexpr int top = FORMAT == STX_E4M3 ? 8 : 15;
    const int e = (int)(most >> 23) - top + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);   // biased by 127 like fp32's
    return most == 0u ? 127u : (uint32_t)max(e, 1);
}
// A scale's value; bytes are 1 to 254.
__device__ inline float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Four numbers as codes, nearest even; what lies above the format's largest number by less than half a step rounds to it.
template <int FORMAT>
__device__ inline uint32_t pack4(float a, float b, float c, float d)
{
    int w = 0;
    if constexpr (FORMAT == STX_E4M3) {
        w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
        w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
    }
    return (uint32_t)w;
}
template <int FORMAT>
__device__ inline void unpack4(uint32_t w, float *v)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    f2 lo, hi;
    if constexpr (FORMAT == STX_E4M3) {
        lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    } else {
        lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false);
        hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
    }
    v[0] = lo.x; v[1] = lo.y; v[2] = hi.x; v[3] = hi.y;
}
// Two numbers over a power of two as codes, nearest even, into the low or the high half of `codes`.  NaN stays NaN; infinities stay
// in E5M2 and become NaN in E4M3.  (These instructions agree with a product and v_cvt_pk_* in every 16-bit number and scale.)
typedef int16_t i16x2_t __attribute__((ext_vector_type(2)));
template <int FORMAT>
__device__ inline i16x2_t code2(i16x2_t codes, float a, float b, float scale, bool high)
{
    if constexpr (FORMAT == STX_E4M3)
        return high ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(codes, a, b, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(codes, a, b, scale, false);
    else
        return high ? __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(codes, a, b, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(codes, a, b, scale, false);
}
template <class T, int FORMAT>
__device__ inline i16x2_t code2(i16x2_t codes, uint32_t pair, float scale, bool high)
{
    if constexpr (__is_same(T, bf16_t)) {
        typedef __bf16 v2_t __attribute__((ext_vector_type(2)));
        const v2_t v = __builtin_bit_cast(v2_t, pair);
        if constexpr (FORMAT == STX_E4M3)
            return high ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(codes, v, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(codes, v, scale, false);
        else
            return high ? __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(codes, v, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(codes, v, scale, false);
    } else {
        typedef _Float16 v2_t __attribute__((ext_vector_type(2)));
        const v2_t v = __builtin_bit_cast(v2_t, pair);
        if constexpr (FORMAT == STX_E4M3)
            return high ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(codes, v, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(codes, v, scale, false);
        else
            return high ? __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(codes, v, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(codes, v, scale, false);
    }
}
template <int FORMAT>
__device__ inline uint32_t code4(float a, float b, float c, float d, float scale)
{
    return __builtin_bit_cast(uint32_t, code2<FORMAT>(code2<FORMAT>(i16x2_t{0, 0}, a, b, scale, false), c, d, scale, true));
}
template <class T, int FORMAT>
__device__ inline uint32_t code4(uint32_t ab, uint32_t cd, float scale)
{
    return __builtin_bit_cast(uint32_t, code2<T, FORMAT>(code2<T, FORMAT>(i16x2_t{0, 0}, ab, scale, false), cd, scale, true));
}
// The codes of an octet.
template <class T, int FORMAT>
__device__ inline uint2 code8(const Octet<T> &o, float scale)
{
    if constexpr (sizeof(T) == 4) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(float, o.w[j]);
        return make_uint2(code4<FORMAT>(v[0], v[1], v[2], v[3], scale), code4<FORMAT>(v[4], v[5], v[6], v[7], scale));
    } else {
        return make_uint2(code4<T, FORMAT>(o.w[0], o.w[1], scale), code4<T, FORMAT>(o.w[2], o.w[3], scale));
    }
}

// A kernel's view of an stx_q8 that it writes (codes null: none).
struct Q8Out {
    uint8_t *codes, *scales;
    int64_t ld, ld_scale;
};

// An octet's codes.
template <class T>
__device__ inline void store_codes(const Q8Out &q, int64_t row, int blk, int l16, uint2 codes)
{
    uint8_t *at = q.codes + row * q.ld + blk * kBlock;
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<uint32_t *>(at + 4 * l16) = codes.x;
        *reinterpret_cast<uint32_t *>(at + 64 + 4 * l16) = codes.y;
    } else {
        *reinterpret_cast<uint2 *>(at + 8 * l16) = codes;
    }
}
// The codes and, by the block's first lane, the scale of an octet as it lies in memory or (with the layout of T) as floats.  All 16
// lanes of the block call it; elements behind the last column are 0 and get codes of 0.
template <class T, int FORMAT>
__device__ inline void store_q8_octet(const Q8Out &q, int64_t row, int blk, int l16, const Octet<T> &o)
{
    const uint32_t byte = block_scale<FORMAT>(row16_max(largest(o)));
    store_codes<T>(q, row, blk, l16, code8<T, FORMAT>(o, scale_of(byte)));
    if (l16 == 0) q.scales[row * q.ld_scale + blk] = (uint8_t)byte;
}
template <class T, int FORMAT>
__device__ inline void store_q8_octet(const Q8Out &q, int64_t row, int blk, int l16, const float (&v)[8])
{
    const uint32_t byte = block_scale<FORMAT>(row16_max(largest<8>(v)));
    const float scale = scale_of(byte);
    store_codes<T>(q, row, blk, l16, make_uint2(code4<FORMAT>(v[0], v[1], v[2], v[3], scale), code4<FORMAT>(v[4], v[5], v[6], v[7], scale)));
    if (l16 == 0) q.scales[row * q.ld_scale + blk] = (uint8_t)byte;
}

}  // namespace stx
