// 8-bit floats and typed row access, shared by the kernels of the 8-bit operators (stx_norm.hip, stx_q8.hip, stx_adamw.hip).
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
// N elements moved down by `by` places of 0 to N, zeros behind them.
template <int N>
__device__ inline void shift_down(float *v, int by)
{
#pragma unroll
    for (int s = N; s >= 1; s >>= 1)
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = (by & s) ? (j + s < N ? v[j + s] : 0.f) : v[j];
}
// The elements of request_octet(row, blk, l16, n) as floats; 0 behind the row's end.
template <class T>
__device__ inline void octet_floats(const Octet<T> &o, int blk, int l16, int64_t n, float (&v)[8])
{
    constexpr int N = 16 / sizeof(T);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (sizeof(T) == 4) v[j] = __builtin_bit_cast(float, o.w[j]);
        else v[j] = to_float<T>((uint16_t)(o.w[j / 2] >> (16 * (j & 1))));
    }
    const int64_t last = octet_pos<T>(blk, l16, 8 - N);
    if (n >= N && __ballot(last + N > n)) {
#pragma unroll
        for (int h = 0; h < 8 / N; ++h) {
            const int64_t over = octet_pos<T>(blk, l16, h * N) + N - n;
            shift_down<N>(v + h * N, (int)(over < 0 ? 0 : over > N ? N : over));
        }
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

// Rounds v to T and, if row is not null, stores it there.
template <class T>
__device__ inline void round_store_octet(T *row, int blk, int l16, int64_t n, float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
        if (!row) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = (int64_t)blk * kBlock + h * 64 + 4 * l16;
            if (at + 4 <= n) {
                const f4u_t q = {v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
                *reinterpret_cast<f4u_t *>(row + at) = q;
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
            *reinterpret_cast<u16x8u_t *>(r16 + at) = q;
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

// The exponent byte of a block's scale from the bits of its largest finite magnitude: both formats' largest numbers are 1.75
// times a power of two, so a magnitude 1.f 2^E needs 2^(E - 8), or one power more where 1.f > 1.75.
template <int FORMAT>
__device__ inline uint32_t block_scale(uint32_t most)
{
    constexpr int top = FORMAT == STX_E4M3 ? 8 : 15;
    const int e = (int)(most >> 23) - top + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);   // biased by 127 like fp32's
    return most == 0u ? 127u : (uint32_t)max(e, 1);
}
// 2^-(byte - 127); byte 1..254
__device__ inline float scale_down(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

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
// A number scaled for its code; an infinity, which E4M3 has not, becomes a NaN.
template <int FORMAT>
__device__ inline float scaled(float v, float down)
{
    if constexpr (FORMAT == STX_E4M3) return abs_bits(v) < kInfBits ? v * down : __builtin_bit_cast(float, 0x7fc00000u);
    return v * down;
}

// A kernel's view of an stx_q8 that it writes (codes null: none).
struct Q8Out {
    uint8_t *codes, *scales;
    int64_t ld, ld_scale;
};

// An octet's codes and, by the block's first lane, its scale.  All 16 lanes of the block call it; elements behind the last
// column are 0 and get codes of 0.
template <class T, int FORMAT>
__device__ inline void store_q8_octet(const Q8Out &q, int64_t row, int blk, int l16, const float (&v)[8])
{
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, finite_bits(v[j]));
    const uint32_t byte = block_scale<FORMAT>(row16_max(most));
    const float down = scale_down(byte);
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = scaled<FORMAT>(v[j], down);
    const uint32_t lo = pack4<FORMAT>(s[0], s[1], s[2], s[3]), hi = pack4<FORMAT>(s[4], s[5], s[6], s[7]);
    uint8_t *at = q.codes + row * q.ld + blk * kBlock;
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<uint32_t *>(at + 4 * l16) = lo;
        *reinterpret_cast<uint32_t *>(at + 64 + 4 * l16) = hi;
    } else {
        *reinterpret_cast<uint2 *>(at + 8 * l16) = make_uint2(lo, hi);
    }
    if (l16 == 0) q.scales[row * q.ld_scale + blk] = (uint8_t)byte;
}

}  // namespace stx
