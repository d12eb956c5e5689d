// AdamW over many tensors, and over the touched rows of a batch's tables, with moments in 32 or in 8 bits.
//
//   m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   p = p - lr decay p;  p = p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Bound by memory: an element of the tables costs 28 bytes with moments in 32 bits and 16 with moments in 8 (p read and written,
// an fp32 gradient read).  Everything is done in one pass: the moments are decoded, stepped and encoded again in registers; a
// block's scale is a maximum over the 16 lanes that hold it.
//
// In 8 bits a rounding to nearest would lose what (1 - b2) g^2 adds whenever it is less than half a code's step, 6 to 12 % of v:
// a v that has to fall or rise slowly would stand still.  So values are rounded up or down at random, in proportion, and the
// average keeps what is added.  v as such, not its root, is what is averaged; STX_E5M2 has the range for it (2^32 within a block).
// Its smallest code stands in for a v that would round to 0, since m, whose range is 2^17, may be large against eps there.
#include "stx_device.h"
#include "stx_emit_body.h"
#include "stx_ops.h"
#include "stx_rowops.h"

namespace stx {

// Tensors of one launch: their descriptions travel as kernel arguments.  4 KB of them, or, for up to 8 tensors, 0.8 KB
// (a call on 6 small ones takes the host 10.4 us with 4 KB, so 9.5).
constexpr int kAdamTensors = 48, kAdamFew = 8;
// Octets of a thread: two (4,000,000 x 128 in 8 bits in 1,320 us, with one in 1,344), or one where workgroups of 4,096 elements
// would leave compute units idle (6 tensors of 34,000 elements in 8 bits: the kernel takes 4.8 us, with two 6.2).
constexpr int adam_tile(int octets) { return kThreads * 8 * octets; }

struct AdamCoef {
    float b1, om1, b2, om2;
    float size, root, eps, decay;          // lr / (1 - b1^t), 1 / sqrt(1 - b2^t), eps, lr * weight_decay
    float gscale;
    uint64_t seed;                         // of this step: the one seeded with it and t 2^16
};
struct AdamHyper {
    double lr, b1, b2;
    AdamCoef k;                            // for the step number that the host knows
    int64_t step;
    const int64_t *step_dev;
    const float *gscale;
};

struct AdamTensorArg {
    float *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    int64_t n;
    uint32_t first;                        // first workgroup of the tensor
    uint16_t g_dtype, flags;
};
template <int N>
struct AdamTensorsArgs {
    AdamHyper h;
    int n, first_tensor;
    AdamTensorArg t[N];
};

// b^t by squaring, in double: the same on the host and here.
__host__ __device__ inline double pow_int(double b, int64_t t)
{
    double r = 1.0;
    for (uint64_t u = (uint64_t)t; u; u >>= 1) {
        if (u & 1u) r *= b;
        b *= b;
    }
    return r;
}
__host__ __device__ inline void set_step(AdamCoef &k, double lr, double b1, double b2, int64_t t)
{
    k.size = (float)(lr / (1.0 - pow_int(b1, t)));
    k.root = (float)(1.0 / sqrt(1.0 - pow_int(b2, t)));
}

__device__ inline AdamCoef coefficients(const AdamHyper &h, uint64_t &step)
{
    AdamCoef k = h.k;
    step = (uint64_t)h.step;
    if (h.step_dev) {
        const int64_t t = max(h.step_dev[0], (int64_t)1);
        set_step(k, h.lr, h.b1, h.b2, t);
        step = (uint64_t)t;
    }
    k.gscale = h.gscale ? h.gscale[0] : 1.0f;
    return k;
}
__device__ inline uint64_t tensor_seed(uint64_t seed, uint64_t step, int tensor)
{
    return splitmix64_at(seed, (step << 16) + (uint64_t)tensor);
}

// One element; every operation rounded once (contraction is off), but the root and the quotient: the instructions
// v_sqrt_f32 and v_rcp_f32 are within a unit of the last place, so the step is within 3 of them, and far below p's own rounding
// when it is small against p.  (Rounded right they take some 25 instructions more: 4,000,000 x 128 in 8 bits 1,469 us, so
// 1,320.)  Both want normal numbers: a small v is scaled, and the host has checked eps.
__device__ inline void adam_element(const AdamCoef &k, float decay, bool scale_g, float &p, float g, float &m, float &v)
{
    if (scale_g) g = g * k.gscale;
    m = m * k.b1 + g * k.om1;
    v = v * k.b2 + (g * g) * k.om2;
    p = p - p * decay;
    const bool small = v < 0x1p-96f;
    const float root = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v) * (small ? k.root * 0x1p-32f : k.root);
    p = p - (m * k.size) * __builtin_amdgcn_rcpf(root + k.eps);
}

// x >= 0 to a format that keeps 23 - DROP bits of the mantissa, up or down by 16 random bits.  The steps below the smallest
// normal number, TINY, are those of the binade that begins there: x is moved into it.
template <int FORMAT>
__device__ inline float round_random(float x, uint32_t noise)
{
    constexpr int DROP = FORMAT == STX_E4M3 ? 20 : 21;
    constexpr float TINY = FORMAT == STX_E4M3 ? 0x1p-6f : 0x1p-14f, TOP = FORMAT == STX_E4M3 ? 448.f : 57344.f;
    const bool low = x < TINY;
    const float z = low ? x + TINY : x;
    const uint32_t b = (__builtin_bit_cast(uint32_t, z) + (noise << (DROP - 16))) & (0xffffffffu << DROP);
    const float q = __builtin_bit_cast(float, b);
    return fminf(low ? q - TINY : q, TOP);
}

// NQ quads of a block as codes, with the block's scale from `most`, the bits of its largest magnitude.  An infinity or a NaN
// among them makes `scale` a NaN.
template <int FORMAT, int NQ>
__device__ inline void encode(const float (&x)[4 * NQ], uint32_t most, const uint32_t (&noise)[4 * NQ], uint32_t (&codes)[NQ], float &scale)
{
    constexpr float TOP = FORMAT == STX_E4M3 ? 448.f : 57344.f;
    const float big = __builtin_bit_cast(float, most);
    const bool live = most >= 0x0d800000u;                                      // 2^-100
    scale = live ? (most < kInfBits ? big * (1.0f / TOP) : __builtin_bit_cast(float, 0x7fc00000u)) : 0.f;
    const float up = (1.0f / big) * TOP;
    float y[4 * NQ];
#pragma unroll
    for (int j = 0; j < 4 * NQ; ++j) {
        y[j] = round_random<FORMAT>(fabsf(x[j]) * up, noise[j]);
        if (FORMAT == STX_E5M2 && y[j] == 0.f && x[j] != 0.f) y[j] = 0x1p-16f;
        y[j] = live ? copysignf(y[j], x[j]) : 0.f;
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) codes[q] = pack4<FORMAT>(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
}

// The random bits of a quad that begins at element `at` (a multiple of 4): m's in the low halves, v's in the high ones.
__device__ inline void quad_noise(uint64_t seed, uint64_t at, uint32_t *m, uint32_t *v)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint64_t u = splitmix64_at(seed, at / 2 + h);
        m[2 * h] = (uint32_t)u & 0xffffu;
        v[2 * h] = (uint32_t)u >> 16;
        m[2 * h + 1] = (uint32_t)(u >> 32) & 0xffffu;
        v[2 * h + 1] = (uint32_t)(u >> 32) >> 16;
    }
}

__device__ inline float load_grad1(const void *g, int dtype, int64_t at)
{
    if (dtype == STX_F32) return ((const float *)g)[at];
    const uint16_t b = ((const uint16_t *)g)[at];
    return dtype == STX_BF16 ? to_float<bf16_t>(b) : to_float<f16_t>(b);
}

// A thread's octets: two quads of a block, 64 elements apart (stx_fp8.h).  Its gradients; 0 for a quad that the end cuts.
template <class T, int O>
__device__ inline void load_grads(const AdamTensorArg &t, int64_t blk0, int l16, float (&g)[O][8])
{
    typedef uint16_t u16x4u_t __attribute__((ext_vector_type(4), aligned(2)));
    using Quad = typename std::conditional<sizeof(T) == 4, f4u_t, u16x4u_t>::type;
    Quad q[O][2];
#pragma unroll
    for (int o = 0; o < O; ++o)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = (blk0 + o * (kThreads / 16)) * kBlock + h * 64 + 4 * l16;
            q[o][h] = Quad{};
            if (at + 4 <= t.n) q[o][h] = *reinterpret_cast<const Quad *>((const T *)t.g + at);
        }
#pragma unroll
    for (int o = 0; o < O; ++o)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (sizeof(T) == 4) g[o][j] = q[o][j / 4][j & 3];
            else g[o][j] = to_float<T>(q[o][j / 4][j & 3]);
        }
}

template <int BITS, int N, int O>
__global__ __launch_bounds__(kThreads) void k_adamw_tensors(AdamTensorsArgs<N> a)
{
    // the tensor of this workgroup: the last one whose first workgroup is not behind it
    const int lane = threadIdx.x & 63;
    const uint32_t first = lane < a.n ? a.t[lane].first : 0xffffffffu;
    const int which = (int)__popcll(__ballot(first <= blockIdx.x)) - 1;
    const AdamTensorArg t = a.t[__builtin_amdgcn_readfirstlane(which)];
    uint64_t step;
    const AdamCoef k = coefficients(a.h, step);
    const float decay = (t.flags & STX_ADAMW_NO_DECAY) ? 0.f : k.decay;
    const bool scale_g = a.h.gscale != nullptr;
    const int l16 = threadIdx.x & 15;
    const int64_t blk0 = (int64_t)(blockIdx.x - t.first) * (adam_tile(O) / kBlock) + (threadIdx.x >> 4);
    using Raw = typename std::conditional<BITS == 32, f4u_t, uint32_t>::type;
    f4u_t pq[O][2];                        // requested first, all of them; a conversion beside a load would wait for it
    Raw mq[O][2], vq[O][2];
    float msq[O], vsq[O];
#pragma unroll
    for (int o = 0; o < O; ++o) {
        const int64_t blk = blk0 + o * (kThreads / 16);
        msq[o] = vsq[o] = 0.f;
        if (BITS == 8 && blk * kBlock < t.n) { msq[o] = t.ms[blk]; vsq[o] = t.vs[blk]; }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = blk * kBlock + h * 64 + 4 * l16;
            pq[o][h] = f4u_t{0.f, 0.f, 0.f, 0.f};
            mq[o][h] = Raw{};
            vq[o][h] = Raw{};
            if (at + 4 <= t.n) {
                pq[o][h] = *reinterpret_cast<const f4u_t *>(t.p + at);
                if constexpr (BITS == 32) {
                    mq[o][h] = *reinterpret_cast<const f4u_t *>((const float *)t.m + at);
                    vq[o][h] = *reinterpret_cast<const f4u_t *>((const float *)t.v + at);
                } else {
                    mq[o][h] = *reinterpret_cast<const u32u_t *>((const uint8_t *)t.m + at);
                    vq[o][h] = *reinterpret_cast<const u32u_t *>((const uint8_t *)t.v + at);
                }
            }
        }
    }
    float p[O][8], m[O][8], v[O][8], g[O][8];
    if (t.g_dtype == STX_F32) load_grads<float, O>(t, blk0, l16, g);
    else if (t.g_dtype == STX_BF16) load_grads<bf16_t, O>(t, blk0, l16, g);
    else load_grads<f16_t, O>(t, blk0, l16, g);
#pragma unroll
    for (int o = 0; o < O; ++o)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float *pp = &p[o][4 * h], *mp = &m[o][4 * h], *vp = &v[o][4 * h];
            if constexpr (BITS == 8) {
                unpack4<STX_E4M3>(mq[o][h], mp);
                unpack4<STX_E5M2>(vq[o][h], vp);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                pp[j] = pq[o][h][j];
                if constexpr (BITS == 32) { mp[j] = mq[o][h][j]; vp[j] = vq[o][h][j]; }
                else { mp[j] *= msq[o]; vp[j] *= vsq[o]; }
            }
        }
    // the end of a tensor of n % 4 != 0 elements, one lane of the tensor
#pragma unroll
    for (int o = 0; o < O; ++o)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = (blk0 + o * (kThreads / 16)) * kBlock + h * 64 + 4 * l16;
            if (at >= t.n || at + 4 <= t.n) continue;
            for (int j = 0; j < 3; ++j) {
                if (at + j >= t.n) continue;
                p[o][4 * h + j] = t.p[at + j];
                g[o][4 * h + j] = load_grad1(t.g, t.g_dtype, at + j);
                if constexpr (BITS == 32) {
                    m[o][4 * h + j] = ((const float *)t.m)[at + j];
                    v[o][4 * h + j] = ((const float *)t.v)[at + j];
                } else {
                    float x[4];
                    unpack4<STX_E4M3>(((const uint8_t *)t.m)[at + j], x);
                    m[o][4 * h + j] = x[0] * msq[o];
                    unpack4<STX_E5M2>(((const uint8_t *)t.v)[at + j], x);
                    v[o][4 * h + j] = x[0] * vsq[o];
                }
            }
        }
    const uint64_t seed = BITS == 8 ? tensor_seed(k.seed, step, a.first_tensor + which) : 0;
#pragma unroll
    for (int o = 0; o < O; ++o) {
        const int64_t blk = blk0 + o * (kThreads / 16);
        if (blk * kBlock >= t.n) break;    // (the lanes of a block together)
#pragma unroll
        for (int j = 0; j < 8; ++j) adam_element(k, decay, scale_g, p[o][j], g[o][j], m[o][j], v[o][j]);
        uint32_t mc[2] = {}, vc[2] = {};
        if constexpr (BITS == 8) {
            uint32_t mm = 0, mv = 0, nm[8], nv[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // (behind the tensor's end: 0 / (0 + eps) with the moments of 0, which no maximum sees)
                mm = max(mm, abs_bits(m[o][j]));
                mv = max(mv, abs_bits(v[o][j]));
            }
            mm = row16_max(mm);
            mv = row16_max(mv);
#pragma unroll
            for (int h = 0; h < 2; ++h) quad_noise(seed, (uint64_t)(blk * kBlock + h * 64 + 4 * l16), nm + 4 * h, nv + 4 * h);
            float ms, vs;
            encode<STX_E4M3, 2>(m[o], mm, nm, mc, ms);
            encode<STX_E5M2, 2>(v[o], mv, nv, vc, vs);
            if (l16 == 0) { t.ms[blk] = ms; t.vs[blk] = vs; }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t at = blk * kBlock + h * 64 + 4 * l16;
            const float *pp = &p[o][4 * h], *mp = &m[o][4 * h], *vp = &v[o][4 * h];
            if (at + 4 <= t.n) {
                *reinterpret_cast<f4u_t *>(t.p + at) = f4u_t{pp[0], pp[1], pp[2], pp[3]};
                if constexpr (BITS == 32) {
                    *reinterpret_cast<f4u_t *>((float *)t.m + at) = f4u_t{mp[0], mp[1], mp[2], mp[3]};
                    *reinterpret_cast<f4u_t *>((float *)t.v + at) = f4u_t{vp[0], vp[1], vp[2], vp[3]};
                } else {
                    *reinterpret_cast<u32u_t *>((uint8_t *)t.m + at) = mc[h];
                    *reinterpret_cast<u32u_t *>((uint8_t *)t.v + at) = vc[h];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (at + j >= t.n) continue;
                    t.p[at + j] = pp[j];
                    if constexpr (BITS == 32) {
                        ((float *)t.m)[at + j] = mp[j];
                        ((float *)t.v)[at + j] = vp[j];
                    } else {
                        ((uint8_t *)t.m)[at + j] = (uint8_t)(mc[h] >> (8 * j));
                        ((uint8_t *)t.v)[at + j] = (uint8_t)(vc[h] >> (8 * j));
                    }
                }
            }
        }
    }
}

// ---- touched rows ------------------------------------------------------------------------------------
struct AdamRowTable {
    float *p;                              // null: the model has no such table
    void *m, *v;
    float *ms, *vs;
    const float *grad;                     // gradient rows, `ld` floats apart, one for each segment
    int32_t d4, mode, number;              // float4 of a row; what follows the update (see k_sgd_rows); number among the tables
};
struct AdamRowsArgs {
    AdamHyper h;
    const int32_t *touched_cols, *n_touched;
    int64_t n_split;                       // columns below: table a; the others: tables b and c
    int ld;
    AdamRowTable a, b, c;
};

// Largest over the lanes that hold a block: 32 of one float4, or the whole row where fewer do.
template <int LPR>
__device__ inline uint32_t block_max(uint32_t v)
{
#pragma unroll
    for (int s = (LPR < 32 ? LPR : 32) / 2; s >= 1; s >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, s, LPR));
    return v;
}

template <int BITS, int LPR, int ITERS>
__device__ inline void adam_row(const AdamCoef &k, uint64_t step, bool scale_g, const AdamRowTable &t, int64_t row, const float *grad, int lig)
{
    const int blocks = (t.d4 + 31) / 32;
    const int64_t base = row * t.d4 * 4;
    using Raw = typename std::conditional<BITS == 32, float4, uint32_t>::type;
    float4 pq[ITERS], gq[ITERS];           // requested first, all of them; lanes behind the row's end request its last float4
    Raw mq[ITERS], vq[ITERS];
    float msq[ITERS], vsq[ITERS];
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int q = min(lig + it * LPR, t.d4 - 1);
        const int64_t at = base + 4 * q;
        pq[it] = ld4(t.p + at);
        gq[it] = ld4_stream(grad + 4 * q);
        if constexpr (BITS == 32) {
            mq[it] = ld4((const float *)t.m + at);
            vq[it] = ld4((const float *)t.v + at);
        } else {
            mq[it] = *reinterpret_cast<const uint32_t *>((const uint8_t *)t.m + at);
            vq[it] = *reinterpret_cast<const uint32_t *>((const uint8_t *)t.v + at);
            msq[it] = t.ms[row * blocks + q / 32];
            vsq[it] = t.vs[row * blocks + q / 32];
        }
    }
    float p[ITERS][4], m[ITERS][4], v[ITERS][4], g[ITERS][4];
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        p[it][0] = pq[it].x; p[it][1] = pq[it].y; p[it][2] = pq[it].z; p[it][3] = pq[it].w;
        g[it][0] = gq[it].x; g[it][1] = gq[it].y; g[it][2] = gq[it].z; g[it][3] = gq[it].w;
        if constexpr (BITS == 32) {
            m[it][0] = mq[it].x; m[it][1] = mq[it].y; m[it][2] = mq[it].z; m[it][3] = mq[it].w;
            v[it][0] = vq[it].x; v[it][1] = vq[it].y; v[it][2] = vq[it].z; v[it][3] = vq[it].w;
        } else {
            const bool in = lig + it * LPR < t.d4;           // (the others' moments are 0: no block's largest is among them)
            unpack4<STX_E4M3>(mq[it], m[it]);
            unpack4<STX_E5M2>(vq[it], v[it]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                m[it][j] = in ? m[it][j] * msq[it] : 0.f;
                v[it][j] = in ? v[it][j] * vsq[it] : 0.f;
                g[it][j] = in ? g[it][j] : 0.f;
            }
        }
    }
    float ss = 0.f;
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            adam_element(k, k.decay, scale_g, p[it][j], g[it][j], m[it][j], v[it][j]);
            if (t.mode == 1) {
                p[it][j] = p[it][j] - floorf(p[it][j]);
                if (p[it][j] >= 1.0f) p[it][j] = 0.0f;
            }
            ss += lig + it * LPR < t.d4 ? p[it][j] * p[it][j] : 0.f;
        }
    if (t.mode == 2) {
        ss = group_sum<LPR>(ss);
        const float inv = ss > 0.f ? 1.0f / sqrtf(ss) : 1.0f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < 4; ++j) p[it][j] *= inv;
    }
    const uint64_t seed = BITS == 8 ? tensor_seed(k.seed, step, t.number) : 0;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int q = lig + it * LPR;
        const int64_t at = base + 4 * q;
        uint32_t mc[1], vc[1];
        if constexpr (BITS == 8) {
            uint32_t mm = 0, mv = 0, nm[4], nv[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) { mm = max(mm, abs_bits(m[it][j])); mv = max(mv, abs_bits(v[it][j])); }
            mm = block_max<LPR>(mm);
            mv = block_max<LPR>(mv);
            quad_noise(seed, (uint64_t)at, nm, nv);
            float ms, vs;
            encode<STX_E4M3, 1>(m[it], mm, nm, mc, ms);
            encode<STX_E5M2, 1>(v[it], mv, nv, vc, vs);
            if (q < t.d4 && q % 32 == 0) {
                t.ms[row * blocks + q / 32] = ms;
                t.vs[row * blocks + q / 32] = vs;
            }
        }
        if (q < t.d4) {
            st4(t.p + at, make_float4(p[it][0], p[it][1], p[it][2], p[it][3]));
            if constexpr (BITS == 32) {
                st4((float *)t.m + at, make_float4(m[it][0], m[it][1], m[it][2], m[it][3]));
                st4((float *)t.v + at, make_float4(v[it][0], v[it][1], v[it][2], v[it][3]));
            } else {
                *reinterpret_cast<uint32_t *>((uint8_t *)t.m + at) = mc[0];
                *reinterpret_cast<uint32_t *>((uint8_t *)t.v + at) = vc[0];
            }
        }
    }
}

template <int BITS, int LPR, int ITERS>
__global__ __launch_bounds__(kThreads) void k_adamw_rows(AdamRowsArgs a)
{
    constexpr int GROUPS = kThreads / LPR;
    const int lig = threadIdx.x % LPR, grp = threadIdx.x / LPR;
    const int32_t U = a.n_touched[0];
    uint64_t step;
    const AdamCoef k = coefficients(a.h, step);
    const bool scale_g = a.h.gscale != nullptr;
    for (int64_t s = (int64_t)blockIdx.x * GROUPS + grp; s < U; s += (int64_t)gridDim.x * GROUPS) {
        const int64_t col = a.touched_cols[s];
        if (col < a.n_split) {
            adam_row<BITS, LPR, ITERS>(k, step, scale_g, a.a, col, a.a.grad + s * a.ld, lig);
        } else {
            if (a.b.p) adam_row<BITS, LPR, ITERS>(k, step, scale_g, a.b, col - a.n_split, a.b.grad + s * a.ld, lig);
            if (a.c.p) adam_row<BITS, LPR, ITERS>(k, step, scale_g, a.c, col - a.n_split, a.c.grad + s * a.ld, lig);
        }
    }
}

// TransR: the matrices of the relations that occur, as rows of kd elements (a multiple of 1,024); a wavefront takes 256 of them.
// Bound by memory (1,345 matrices of 128 x 128: 90 us with moments in 32 bits, 617 MB, and 62 in 8, 353 MB; a part stays in the caches).
struct AdamProjArgs {
    AdamHyper h;
    const int32_t *touched_cols, *n_touched, *first_rel_seg;
    int32_t n_ent;
    int64_t kd;
    AdamRowTable t;                        // p, m, v, ms, vs, number; grad: dL/dM_r, as the matrices
};
template <int BITS>
__global__ __launch_bounds__(kThreads) void k_adamw_proj(AdamProjArgs a)
{
    const int32_t U = a.n_touched[0], target = a.n_ent + (int32_t)blockIdx.x;
    int32_t lo = a.first_rel_seg[0], hi = U;                 // relation columns sort after all entity columns
    while (lo < hi) {                                        // first position with touched_cols[pos] >= target
        const int32_t mid = (lo + hi) >> 1;
        if (a.touched_cols[mid] < target) lo = mid + 1; else hi = mid;
    }
    if (lo >= U || a.touched_cols[lo] != target) return;
    uint64_t step;
    const AdamCoef k = coefficients(a.h, step);
    // (as a row of 64 float4 of a table of such rows: blocks of 128 are whole in it)
    const int64_t row = ((int64_t)blockIdx.x * a.kd + (int64_t)blockIdx.y * kThreads * 4) / 256 + (threadIdx.x >> 6);
    adam_row<BITS, 64, 1>(k, step, a.h.gscale != nullptr, a.t, row, a.t.grad + row * 256, threadIdx.x & 63);
}

// ---- dispatch ------------------------------------------------------------------------------------------
static AdamHyper make_hyper(const stx_adamw *h)
{
    AdamHyper a{};
    a.lr = h->lr; a.b1 = h->beta1; a.b2 = h->beta2;
    a.k.b1 = (float)h->beta1; a.k.om1 = (float)(1.0 - h->beta1);
    a.k.b2 = (float)h->beta2; a.k.om2 = (float)(1.0 - h->beta2);
    a.k.eps = (float)h->eps;
    a.k.decay = (float)(h->lr * h->weight_decay);
    a.k.gscale = 1.0f;
    a.k.seed = h->seed;
    if (!h->step_dev) set_step(a.k, h->lr, h->beta1, h->beta2, h->step);
    a.step = h->step;
    a.step_dev = h->step_dev;
    a.gscale = h->grad_scale;
    return a;
}

// Tensors from number i on, as many as one launch takes; false: all of them empty.
template <int N, int O>
static bool adam_tensors_go(stx_ctx *c, const stx_adamw *h, const stx_adamw_tensor *tensors, int n, int &i)
{
    AdamTensorsArgs<N> a;
    static_assert(sizeof(a) <= 4096, "kernel arguments");
    a.h = make_hyper(h);
    a.n = 0;
    a.first_tensor = i;
    uint64_t blocks = 0;
    for (; i < n && a.n < N; ++i) {
        const stx_adamw_tensor &t = tensors[i];
        const uint64_t need = ((uint64_t)t.n + adam_tile(O) - 1) / adam_tile(O);
        if (blocks + need > (uint64_t)kMaxItems / kThreads) break;     // (the C entry has checked that one tensor fits)
        // (an empty tensor shares its first workgroup with the next one, which the search finds)
        a.t[a.n++] = {t.p, t.g, t.s.m, t.s.v, t.s.m_scale, t.s.v_scale, t.n, (uint32_t)blocks, (uint16_t)t.g_dtype, (uint16_t)t.flags};
        blocks += need;
    }
    if (!blocks) return false;
    ProfScope prof(c, "k_adamw_tensors");
    if (h->bits == 8) hipLaunchKernelGGL((k_adamw_tensors<8, N, O>), dim3((unsigned)blocks), dim3(kThreads), 0, c->stream, a);
    else hipLaunchKernelGGL((k_adamw_tensors<32, N, O>), dim3((unsigned)blocks), dim3(kThreads), 0, c->stream, a);
    return true;
}

stx_status launch_adamw_tensors(stx_ctx *c, const stx_adamw *h, const stx_adamw_tensor *tensors, int n)
{
    uint64_t full = 0;
    for (int i = 0; i < n && full < 256; ++i) full += ((uint64_t)tensors[i].n + adam_tile(2) - 1) / adam_tile(2);
    auto *go = n <= kAdamFew ? full < 256 ? adam_tensors_go<kAdamFew, 1> : adam_tensors_go<kAdamFew, 2>
                             : full < 256 ? adam_tensors_go<kAdamTensors, 1> : adam_tensors_go<kAdamTensors, 2>;
    bool launched = false;
    for (int i = 0; i < n;) launched |= go(c, h, tensors, n, i);
    return launched ? hip_ok(hipGetLastError()) : STX_OK;
}

template <int LPR, int ITERS>
static void adam_rows_go(stx_ctx *c, const stx_incidence *inc, int bits, const AdamRowsArgs &a)
{
    constexpr int GROUPS = kThreads / LPR;
    const int64_t ncol = c->cfg.n_ent + c->cfg.n_rel, cap = inc->nnz < ncol ? inc->nnz : ncol;
    int64_t blocks = (cap + GROUPS - 1) / GROUPS;
    if (blocks > 8192) blocks = 8192;
    ProfScope prof(c, "k_adamw_rows");
    if (bits == 8) hipLaunchKernelGGL((k_adamw_rows<8, LPR, ITERS>), dim3((unsigned)blocks), dim3(kThreads), 0, c->stream, a);
    else hipLaunchKernelGGL((k_adamw_rows<32, LPR, ITERS>), dim3((unsigned)blocks), dim3(kThreads), 0, c->stream, a);
}

stx_status launch_adamw_step(stx_ctx *c, stx_params *p, const stx_incidence *inc, const stx_grads *g, const stx_adamw *h,
                             const stx_adamw_state *s)
{
    if (inc->n_rows == 0) return STX_OK;
    const int dim = c->cfg.dim;
    const bool stacked = c->cfg.model == STX_TRANSE || c->cfg.model == STX_TORUSE, transh = c->cfg.model == STX_TRANSH;
    const bool transr = c->cfg.model == STX_TRANSR;
    auto table = [](float *t, const stx_moments &m, const float *grad, int width, int mode, int number) {
        return AdamRowTable{t, m.m, m.v, m.m_scale, m.v_scale, grad, width / 4, mode, number};
    };
    AdamRowsArgs a{};
    a.h = make_hyper(h);
    a.touched_cols = inc->at_touched_cols;
    a.n_touched = inc->n_touched;
    a.ld = c->ld;
    a.n_split = stacked ? c->cfg.n_ent + c->cfg.n_rel : c->cfg.n_ent;
    a.a = table(p->ent, s->ent, g->rows, dim, c->cfg.model == STX_TORUSE ? 1 : 0, 0);
    if (!stacked) a.b = table(p->rel, s->rel, g->rows, c->cfg.rel_dim, 0, 1);
    if (transh) a.c = table(p->w, s->w, g->w_rows, dim, (c->cfg.flags & STX_FLAG_RENORM_W) ? 2 : 0, 2);
    const Launch L = row_launch(c->ld);
    STX_DISPATCH_ROW(L, adam_rows_go, c, inc, h->bits, a);
    if (transr) {
        AdamProjArgs m{};
        m.h = a.h;
        m.touched_cols = inc->at_touched_cols;
        m.n_touched = inc->n_touched;
        m.first_rel_seg = inc->at_seg_id + 2 * inc->n_rows;
        m.n_ent = (int32_t)c->cfg.n_ent;
        m.kd = (int64_t)c->cfg.rel_dim * dim;
        m.t = table(p->proj, s->proj, g->proj, 256, 0, 3);
        const dim3 grid((unsigned)c->cfg.n_rel, (unsigned)(m.kd / (kThreads * 4)));
        ProfScope prof(c, "k_adamw_proj");
        if (h->bits == 8) hipLaunchKernelGGL(k_adamw_proj<8>, grid, dim3(kThreads), 0, c->stream, m);
        else hipLaunchKernelGGL(k_adamw_proj<32>, grid, dim3(kThreads), 0, c->stream, m);
    }
    return hip_ok(hipGetLastError());
}

}  // namespace stx
