// C = A B^T of matrices held in 8 bits, a power of two for each block of 128 columns of a row.
//
//   C[i][j] = sum over blocks of 2^(ea[i][b] + eb[j][b]) sum over the block's 128 columns of a[i][k] b[j][k]
//
// Two ways through the matrix cores, by what the output keeps:
//
//   16-bit outputs: v_mfma_scale_*_f8f6f4 on the codes, which takes the powers of two itself (a byte per 32 columns and row, here
//   the same one four times).  It sums its products in eights, and in each eight what lies below 2^-13 of the largest is cut
//   off: 1.4e-5 of the result for normal data (2-norm), whatever the length; an output of bf16 rounds by 1.7e-3, of fp16 by 2.1e-4.
//   (The unscaled 8-bit instructions cut in the same place.)
//
//   fp32 outputs: codes become bfloat16 times their power of two (v_cvt_scalef32_pk_bf16_*: exact, two codes an instruction) in
//   front of v_mfma_f32_*_bf16, whose products are whole: 1e-7 of the result, at half the rate.  The conversions go on beside the
//   matrix instructions (three to one of 32 x 32 x 16 make it 5 % longer).  Powers of two that take codes out of bfloat16's normal
//   numbers cannot go into them: a wavefront that meets one moves a power of two from all its rows of A to those of B, for that block
//   (balance); where there is none that suits all of them, it forms its sums anew in the end, without any in the operands (sums_far).
//   Watching for them takes 9 instructions a stage.
//
// Times below are of calls in a row after 0.15 s of the same; cards differ by 6 %.  For some 10 ms after a rest the card lowers its
// clock, and large products take up to 30 % longer; what then prefers another way than afterwards is said with both.
#include "stx_device.h"
#include "stx_ops.h"

namespace stx {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct MmArgs {
    const uint8_t *a, *as, *b, *bs;
    int64_t lda, ldas, ldb, ldbs;
    int64_t m, n;
    int nkb;                               // blocks of 128 columns
    int kb_split;                          // blocks of a slice (a multiple of 4), of `splits` slices
    int splits;
    int ntm, ntn;
    void *out;                             // splits > 1: fp32 [split][m][n] instead, with ldo = n
    int64_t ldo;
    int dtype;
    int past;                              // fp32 and bf16 outputs go past the caches (launch_q8_matmul); fp16 ones never do
};

template <int FORMAT>
__device__ inline bf16x2_t widen2(int w, float scale, bool hi)
{
    if constexpr (FORMAT == STX_E4M3) return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    else return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, false);
}
// Scales with which every code but 0 becomes a normal bfloat16: E4M3's are 2^-9 to 448, E5M2's 2^-16 to 57344.
template <int FORMAT> constexpr int kLeast = FORMAT == STX_E4M3 ? 10 : 17;
template <int FORMAT> constexpr int kMost = FORMAT == STX_E4M3 ? 246 : 239;
template <int FORMAT, int N>
__device__ inline bool in_reach(const uint32_t (&bytes)[N])
{
    uint32_t above = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) above = max(above, bytes[i] - kLeast<FORMAT>);
    return above <= uint32_t(kMost<FORMAT> - kLeast<FORMAT>);
}
// Least and largest of a wavefront's scales.
template <int N>
__device__ inline void range_of(const uint32_t (&bytes)[N], int &least, int &most)
{
    least = most = (int)bytes[0];
#pragma unroll
    for (int i = 1; i < N; ++i) { least = min(least, (int)bytes[i]); most = max(most, (int)bytes[i]); }
    for (int d = 32; d >= 1; d >>= 1) { least = min(least, __shfl_xor(least, d, 64)); most = max(most, __shfl_xor(most, d, 64)); }
}
// The scales of a block, of which some are out of reach, with a power of two moved from A to B that brings all into it; false if there
// is none.  The products stay what they are.
template <int FA, int FB, int MI, int NI>
__device__ inline bool balance(uint32_t (&a)[MI], uint32_t (&b)[NI])
{
    int a0, a1, b0, b1;
    range_of(a, a0, a1);
    range_of(b, b0, b1);
    const int low = max(kLeast<FA> - a0, b1 - kMost<FB>), high = min(kMost<FA> - a1, b0 - kLeast<FB>), move = min(max(low, 0), high);
    if (low > high) return false;
#pragma unroll
    for (int i = 0; i < MI; ++i) a[i] += move;
#pragma unroll
    for (int j = 0; j < NI; ++j) b[j] -= move;
    return true;
}

template <int FORMAT>
__device__ inline bf16x8_t widen8(int lo, int hi, float scale)
{
    const bf16x2_t a = widen2<FORMAT>(lo, scale, false), b = widen2<FORMAT>(lo, scale, true);
    const bf16x2_t c = widen2<FORMAT>(hi, scale, false), d = widen2<FORMAT>(hi, scale, true);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Four consecutive outputs of a row.
__device__ inline void store4(const MmArgs &p, int split, int64_t i, int64_t j, const f32x4_t v)
{
    if (i >= p.m || j >= p.n) return;
    const int64_t at = ((int64_t)split * p.m + i) * p.ldo + j;
    const bool whole = j + 4 <= p.n;
    if (p.dtype == STX_F32) {
        float *o = (float *)p.out + at;
        if (whole) *reinterpret_cast<f4u_t *>(o) = f4u_t{v[0], v[1], v[2], v[3]};
        else
            for (int r = 0; r < 4 && j + r < p.n; ++r) o[r] = v[r];
        return;
    }
    typedef uint16_t u16x4u_t __attribute__((ext_vector_type(4), aligned(2)));
    u16x4u_t h;
#pragma unroll
    for (int r = 0; r < 4; ++r) h[r] = p.dtype == STX_BF16 ? from_float<bf16_t>(v[r]) : from_float<f16_t>(v[r]);
    uint16_t *o = (uint16_t *)p.out + at;
    if (whole) *reinterpret_cast<u16x4u_t *>(o) = h;
    else
        for (int r = 0; r < 4 && j + r < p.n; ++r) o[r] = h[r];
}

// Tile number `number`: every die takes a run of consecutive tiles (workgroups go round the dies in turn), along stripes of
// kStripe tiles of A, so that what a die reads at a time fits its L2.
constexpr int kDies = 8, kStripe = 8;
__device__ inline void tile_of(const MmArgs &p, unsigned number, unsigned total, int &tm, int &tn, int &split)
{
    const unsigned die = number % kDies, each = total / kDies, more = total % kDies;
    const unsigned i = die * each + (die < more ? die : more) + number / kDies;
    const unsigned tiles = (unsigned)p.ntm * (unsigned)p.ntn;
    split = __builtin_amdgcn_readfirstlane((int)(i / tiles));
    const unsigned t = i % tiles, stripe = t / (unsigned)(kStripe * p.ntn), r = t % (unsigned)(kStripe * p.ntn);
    const unsigned first = stripe * kStripe, high = min((unsigned)kStripe, (unsigned)p.ntm - first);
    tm = __builtin_amdgcn_readfirstlane((int)(first + r % high));
    tn = __builtin_amdgcn_readfirstlane((int)(r / high));
}

typedef const __attribute__((address_space(1))) void *global_ptr_t;
typedef __attribute__((address_space(3))) void *lds_ptr_t;

typedef float f32x16_t __attribute__((ext_vector_type(16)));

template <int FA, int FB>
__device__ inline f32x16_t multiply32(const i32x4_t *b, uint32_t scale_b, const i32x4_t *a, uint32_t scale_a, f32x16_t acc)
{
    const i32x8_t av = {a[0][0], a[0][1], a[0][2], a[0][3], a[1][0], a[1][1], a[1][2], a[1][3]};
    const i32x8_t bv = {b[0][0], b[0][1], b[0][2], b[0][3], b[1][0], b[1][1], b[1][2], b[1][3]};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bv, av, acc, FB, FA, 0, (int)scale_b, 0, (int)scale_a);
}

// Conversions and scalars may cross, nothing else.
__device__ inline void keep_order() { __builtin_amdgcn_sched_barrier(0x6); }

// A wavefront's sums over blocks kb, kb + step, ... of rows from i0 of A and j0 of B, straight from memory, whatever the scales: a
// block's sum is formed of the codes as they are, and takes its power of two as it is added.  SIZE 32 or 16: that of a product.
template <int FA, int FB, int SIZE, int MI, int NI, class V>
__device__ inline void sums_far(const MmArgs &p, int64_t i0, int64_t j0, int kb, int end, int step, V (&acc)[MI][NI])
{
    constexpr int GROUPS = 64 / SIZE, REGS = SIZE * SIZE / 64;           // lanes of a row; sums of a lane
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int in = lane % SIZE, group = lane / SIZE;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = V{};
    for (; kb < end; kb += step) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int64_t ra = min(i0 + i * SIZE + in, p.m - 1), rb = min(j0 + j * SIZE + in, p.n - 1);
                V t{};
#pragma unroll
                for (int u = 0; u < 8 / GROUPS; ++u) {       // 16 codes a lane
                    const int at = kb * kBlock + (u * GROUPS + group) * 16;
                    const i32x4_t a = *reinterpret_cast<const i32x4_t *>(p.a + ra * p.lda + at), b = *reinterpret_cast<const i32x4_t *>(p.b + rb * p.ldb + at);
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const bf16x8_t wa = widen8<FA>(a[2 * s], a[2 * s + 1], 1.0f), wb = widen8<FB>(b[2 * s], b[2 * s + 1], 1.0f);
                        if constexpr (SIZE == 32) t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb, wa, t, 0, 0, 0);
                        else t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, wa, t, 0, 0, 0);
                    }
                    asm volatile("" ::: "memory");           // one after the other: the registers are the hot loop's
                    __builtin_amdgcn_sched_barrier(0);
                }
                const int ea = p.as[ra * p.ldas + kb] - 254, eb = p.bs[rb * p.ldbs + kb];
#pragma unroll
                for (int r = 0; r < REGS; ++r)               // (a lane holds one row of A, and of B rows in fours)
                    acc[i][j][r] += __builtin_ldexpf(t[r], ea + __shfl(eb, r / 4 * 4 * GROUPS + group * 4 + r % 4, SIZE));
                asm volatile("" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
            }
    }
}

// The products of a wavefront's step: 32 codes a lane and fragment.  between(u) is called after each of 2 MI parts of them.
template <bool WIDE, int FA, int FB, int MI, int NI, class F>
__device__ inline void multiply_step(const i32x4_t (&a)[MI][2], const uint32_t (&sca)[MI], const i32x4_t (&b)[NI][2], const uint32_t (&scb)[NI],
                                     f32x16_t (&acc)[MI][NI], F between)
{
    static_assert(NI == 2, "parts");
    if constexpr (!WIDE) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                acc[i][j] = multiply32<FA, FB>(b[j], scb[j], a[i], sca[i], acc[i][j]);
                between(i * NI + j);
            }
    } else {
        // A fragment's conversions stand between the products before its own, two or three of theirs to a product (left to the compiler
        // they gather where the products end: 14,951 x 1,024 over 8,192 columns takes 2 % longer)
        bf16x8_t wb[2][NI][2], wa[2][2];
        auto widen_a = [&](int u, int s) { wa[u & 1][s] = widen8<FA>(a[u % MI][u / MI][2 * s], a[u % MI][u / MI][2 * s + 1], scale_of(sca[u % MI])); };
        auto widen_b = [&](int h, int j, int s) { wb[h][j][s] = widen8<FB>(b[j][h][2 * s], b[j][h][2 * s + 1], scale_of(scb[j])); };
        widen_b(0, 0, 0);
        widen_a(0, 0);
#pragma unroll
        for (int u = 0; u < 2 * MI; ++u) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int s = q >> 1, j = q & 1, i = u % MI, h = u / MI;
                if (u == 0 && q == 1) widen_b(0, 1, 0);
                if (u == 0 && q == 2) { widen_b(0, 0, 1); widen_a(0, 1); }
                if (u == 0 && q == 3) widen_b(0, 1, 1);
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[h][j][s], wa[u & 1][s], acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if (q & 1) { if (u + 1 < 2 * MI) widen_a(u + 1, q >> 1); }
                else if (u < MI) {
                    if (MI == 2 && u == 1) { widen_b(1, 0, q >> 1); widen_b(1, 1, q >> 1); }
                    if (MI == 4 && u >= 2) widen_b(1, q >> 1, u - 2);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            between(u);
        }
    }
#pragma unroll
    for (int i = 0; i < MI; ++i)           // (pins the products to this place)
#pragma unroll
        for (int j = 0; j < NI; ++j) asm volatile("" : "+v"(acc[i][j]));
}

// A step's fragments, 4 KB apart in LDS, from a and b with their halves at a0 / a1 and b0 / b1; and their scales.  Every read of LDS
// stands in one block with its wait: the compiler would put waits for the codes under way before them.
__device__ inline void read_step(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1, i32x4_t (&a)[4][2], i32x4_t (&b)[2][2])
{
    asm volatile("ds_read_b128 %0, %12\n\tds_read_b128 %1, %13\n\t"
                 "ds_read_b128 %2, %12 offset:4096\n\tds_read_b128 %3, %13 offset:4096\n\t"
                 "ds_read_b128 %4, %14\n\tds_read_b128 %5, %15\n\t"
                 "ds_read_b128 %6, %14 offset:4096\n\tds_read_b128 %7, %15 offset:4096\n\t"
                 "ds_read_b128 %8, %14 offset:8192\n\tds_read_b128 %9, %15 offset:8192\n\t"
                 "ds_read_b128 %10, %14 offset:12288\n\tds_read_b128 %11, %15 offset:12288\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(b[0][0]), "=&v"(b[0][1]), "=&v"(b[1][0]), "=&v"(b[1][1]), "=&v"(a[0][0]), "=&v"(a[0][1]), "=&v"(a[1][0]),
                   "=&v"(a[1][1]), "=&v"(a[2][0]), "=&v"(a[2][1]), "=&v"(a[3][0]), "=&v"(a[3][1])
                 : "v"(b0), "v"(b1), "v"(a0), "v"(a1) : "memory");
}
__device__ inline void read_step(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1, i32x4_t (&a)[2][2], i32x4_t (&b)[2][2])
{
    asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %9\n\t"
                 "ds_read_b128 %2, %8 offset:4096\n\tds_read_b128 %3, %9 offset:4096\n\t"
                 "ds_read_b128 %4, %10\n\tds_read_b128 %5, %11\n\t"
                 "ds_read_b128 %6, %10 offset:4096\n\tds_read_b128 %7, %11 offset:4096\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(b[0][0]), "=&v"(b[0][1]), "=&v"(b[1][0]), "=&v"(b[1][1]), "=&v"(a[0][0]), "=&v"(a[0][1]), "=&v"(a[1][0]),
                   "=&v"(a[1][1])
                 : "v"(b0), "v"(b1), "v"(a0), "v"(a1) : "memory");
}
__device__ inline void read_scales(uint32_t at_a, uint32_t at_b, uint32_t (&a)[4], uint32_t (&b)[2])
{
    asm volatile("ds_read_u8 %0, %6\n\tds_read_u8 %1, %6 offset:128\n\tds_read_u8 %2, %6 offset:256\n\t"
                 "ds_read_u8 %3, %6 offset:384\n\tds_read_u8 %4, %7\n\tds_read_u8 %5, %7 offset:128\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a[0]), "=&v"(a[1]), "=&v"(a[2]), "=&v"(a[3]), "=&v"(b[0]), "=&v"(b[1]) : "v"(at_a), "v"(at_b) : "memory");
}
__device__ inline void read_scales(uint32_t at_a, uint32_t at_b, uint32_t (&a)[2], uint32_t (&b)[2])
{
    asm volatile("ds_read_u8 %0, %4\n\tds_read_u8 %1, %4 offset:128\n\tds_read_u8 %2, %5\n\tds_read_u8 %3, %5 offset:128\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a[0]), "=&v"(a[1]), "=&v"(b[0]), "=&v"(b[1]) : "v"(at_a), "v"(at_b) : "memory");
}

// Nothing moves across: neither memory accesses nor matrix instructions.
__device__ inline void phase_end()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// N consecutive outputs of a row.  PAST: stored past the caches.
template <int N, bool PAST, class T, class V>
__device__ inline void store_piece(T *out, const MmArgs &p, int split, int64_t i, int64_t j, const V v)
{
    if (i >= p.m || j >= p.n) return;
    T *o = out + ((int64_t)split * p.m + i) * p.ldo + j;
    if (j + N <= p.n) {
        if (PAST) __builtin_nontemporal_store(v, reinterpret_cast<V *>(o));
        else *reinterpret_cast<V *>(o) = v;
        return;
    }
#pragma unroll
    for (int r = 0; r < N; ++r)
        if (j + r < p.n) o[r] = v[r];
}

// Between LDS accesses of all wavefronts; stores stay under way.
__device__ inline void leave_sync()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// A workgroup's outputs turn in LDS, so that its rows leave whole: as they stand, a store would have 16 bytes of 32 rows.  PASSES
// parts of a wavefront's rows after each other, so many as NW * 8 KB need.  Pieces of 16 bytes are permuted by the row.  All
// wavefronts call it, when nothing else of that LDS is in use; their own requests have arrived before the first store, which a
// wait for them would wait for too.  (LDS by instructions of its own: the compiler would wait for all requests before them.)
template <class T, bool PAST, int BM, int BN, int WM, int WN, int MI, int NI>
__device__ inline void leave_as(const MmArgs &p, int split, int64_t m0, int64_t n0, const f32x16_t (&acc)[MI][NI], uint32_t lds)
{
    constexpr int PASSES = BM * BN * sizeof(T) / (WM * WN * 8192), ROWS = BM / PASSES, PART = MI / PASSES, LINE = BN * sizeof(T), PIECES = LINE / 16;
    constexpr int PER = 1024 / LINE, NW = WM * WN;           // rows of a wavefront's store
    static_assert(ROWS == 8 * NW * PER, "eight stores of a wavefront a pass");
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));         // (no address of these is kept through the products)
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), l31 = lane & 31, half = lane >> 5;
    const int wm = wave % WM, wn = wave / WM * (BN / WN);
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        if (pass) leave_sync();
#pragma unroll
        for (int i = 0; i < PART; ++i) {
            const uint32_t line = lds + ((wm * PART + i) * 32 + l31) * LINE;
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x16_t &v = acc[pass * PART + i][j];
                    const int byte = (wn + j * 32 + q * 8 + half * 4) * (int)sizeof(T);
                    const uint32_t at = line + ((byte >> 4) ^ (l31 & 15)) * 16 + (byte & 15);
                    if constexpr (sizeof(T) == 4) {
                        const f32x4_t four = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                        asm volatile("ds_write_b128 %0, %1" :: "v"(at), "v"(four) : "memory");
                    } else {
                        typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
                        u32x2_t four;
#pragma unroll
                        for (int r = 0; r < 2; ++r)
                            four[r] = from_float<T>(v[4 * q + 2 * r]) | (uint32_t)from_float<T>(v[4 * q + 2 * r + 1]) << 16;
                        asm volatile("ds_write_b64 %0, %1" :: "v"(at), "v"(four) : "memory");
                    }
                }
        }
        if (pass == 0) __builtin_amdgcn_s_waitcnt(0x0f70);
        leave_sync();
        const int r0 = wave * PER + lane / PIECES, c = lane % PIECES;           // rows r0, r0 + NW * PER, ...
        i32x4_t v[8];
        asm volatile("ds_read_b128 %0, %8\n\tds_read_b128 %1, %8 offset:%9\n\tds_read_b128 %2, %8 offset:%10\n\t"
                     "ds_read_b128 %3, %8 offset:%11\n\tds_read_b128 %4, %8 offset:%12\n\tds_read_b128 %5, %8 offset:%13\n\t"
                     "ds_read_b128 %6, %8 offset:%14\n\tds_read_b128 %7, %8 offset:%15\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
                     : "v"(lds + r0 * LINE + c * 16), "n"(NW * 1024), "n"(2 * NW * 1024), "n"(3 * NW * 1024), "n"(4 * NW * 1024),
                       "n"(5 * NW * 1024), "n"(6 * NW * 1024), "n"(7 * NW * 1024) : "memory");
#pragma unroll
        for (int it = 0; it < 8; ++it) {
            const int lr = it * NW * PER + r0, at = c ^ (lr & 15);
            const int64_t row = m0 + (lr / (PART * 32)) * (BM / WM) + pass * (PART * 32) + lr % (PART * 32);
            if constexpr (sizeof(T) == 4) store_piece<4, PAST>((float *)p.out, p, split, row, n0 + at * 4, __builtin_bit_cast(f4u_t, v[it]));
            else store_piece<8, PAST>((uint16_t *)p.out, p, 0, row, n0 + at * 8, __builtin_bit_cast(u16x8u_t, v[it]));
        }
    }
}
template <bool WIDE, int BM, int BN, int WM, int WN, int MI, int NI>
__device__ inline void leave(const MmArgs &p, int split, int64_t m0, int64_t n0, const f32x16_t (&acc)[MI][NI], uint32_t lds)
{
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");       // the last products are whole (the compiler knows no reads of an asm block)
    if (WIDE || p.dtype == STX_F32) {
        if (p.past) leave_as<float, true, BM, BN, WM, WN>(p, split, m0, n0, acc, lds);
        else leave_as<float, false, BM, BN, WM, WN>(p, split, m0, n0, acc, lds);
    } else if (p.dtype == STX_BF16) {
        if (p.past) leave_as<bf16_t, true, BM, BN, WM, WN>(p, split, m0, n0, acc, lds);
        else leave_as<bf16_t, false, BM, BN, WM, WN>(p, split, m0, n0, acc, lds);
    } else {                               // (no kernel of its own for fp16 past the caches)
        leave_as<f16_t, false, BM, BN, WM, WN>(p, split, m0, n0, acc, lds);
    }
}

// A BM x BN tile by WM x WN wavefronts, in 32 x 32 products.  A stage is one block of 128 columns: its codes go straight to LDS, a
// row's 128 bytes in a line (requested as one), and a stage is multiplied in two steps of 64 columns while the next one's codes are
// under way into the other buffer.  Piece c (16 bytes) of row r lies at c ^ (r / 2 % 8), and a lane reads pieces h and h + 2 of its
// row's half, h = lane / 32: 2.86 ns a read and CU, as 64 lanes side by side; other orders 3.6 to 7.0.
//
// Four wavefronts: a workgroup takes half of a CU, so that one's outputs leave while the other multiplies.  Eight: two of them
// share a SIMD, and the second runs one phase behind the first (it passes one more barrier at the start), so that one multiplies
// while the other reads its fragments and requests codes:
//
//   phase      4s             4s + 1         4s + 2         4s + 3
//   group 0    read 1st       multiply 1st   read 2nd       multiply 2nd
//   group 1    multiply 2nd   read 1st       multiply 1st   read 2nd
//
// (of stage s; group 1 still multiplies s - 1 in phase 4s).  A stage's codes of A are requested beside the first reads of the stage
// before, when everybody has read their buffer, those of B, which only one group reads, between that group's products two stages
// before.  (All of them beside the reads, from 64-bit addresses, made those phases the longest: 8,192 x 8,192 x 8,192 took 8 % longer.)
// Every wavefront waits for its own at the end of 4s + 3, before the first read of the next stage; group 0 leaves those in
// flight that it has just requested.
//
// One workgroup for each compute unit takes every 256th tile, and requests the next one's first stage before its outputs leave (4,096 x
// 14,951 bf16 over 1,024 columns in 78 to 84 us, 7 % longer with a workgroup for each tile).
template <int BM, int BN, int WM, int WN, bool WIDE, int FA, int FB>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_q8_mm(MmArgs p)
{
    constexpr int NW = WM * WN, MI = BM / WM / 32, NI = BN / WN / 32, LA = BM / 8 / NW, LB = BN / 8 / NW, BUF = (BM + BN) * kBlock;
    constexpr bool PHASES = NW == 8;
    constexpr int ROOM = NW * 8192;        // what the outputs turn in, from the second buffer on
    static_assert(BM + BN <= NW * 64, "a thread for each row's scales");
    __shared__ __align__(16) uint8_t s_buf[BUF + (BUF > ROOM ? BUF : ROOM)];
    __shared__ uint32_t s_scale[2][BM + BN];                 // a word for four stages
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int l31 = lane & 31, half = lane >> 5, group = wave >> 2;
    // requests: a wavefront's 64 pieces are 8 rows, of B the rows that its group reads; rows behind the last one repeat it.  Offsets of
    // 32 bits to a scalar base: a 64-bit sum in a vector register would wait until the other group's products are done
    const int piece = ((lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7)) * 16;
    constexpr int NG = PHASES ? 4 : NW;    // wavefronts of a group
    const int b_first = PHASES ? group * (BN / 16) + (wave & 3) : wave;         // in eights of rows
    const bool of_a = wave * 64 < BM;      // whose rows' scales this wavefront requests
    uint32_t oa[LA], ob[LB], os;
    const uint8_t *ga, *gb, *gs;
    int64_t m0, n0;
    int split, stages;
    auto aim = [&](unsigned number, unsigned total) {
        int tm, tn, l8 = lane >> 3, thread = threadIdx.x;
        asm volatile("" : "+v"(l8), "+v"(thread));
        tile_of(p, number, total, tm, tn, split);
        m0 = (int64_t)tm * BM;
        n0 = (int64_t)tn * BN;
        const int kb0 = split * p.kb_split;
        stages = min(kb0 + p.kb_split, p.nkb) - kb0;
#pragma unroll
        for (int i = 0; i < LA; ++i) oa[i] = (uint32_t)(min((int64_t)((i * NW + wave) * 8 + l8), p.m - 1 - m0) * p.lda) + piece;
#pragma unroll
        for (int i = 0; i < LB; ++i) ob[i] = (uint32_t)(min((int64_t)((i * NG + b_first) * 8 + l8), p.n - 1 - n0) * p.ldb) + piece;
        ga = p.a + m0 * p.lda + (int64_t)kb0 * kBlock;
        gb = p.b + n0 * p.ldb + (int64_t)kb0 * kBlock;
        gs = (of_a ? p.as + m0 * p.ldas : p.bs + n0 * p.ldbs) + kb0;
        os = of_a ? (uint32_t)(min((int64_t)thread, p.m - 1 - m0) * p.ldas) : (uint32_t)(min((int64_t)thread - BM, p.n - 1 - n0) * p.ldbs);
    };
    auto request = [&](const uint8_t *from, uint32_t &at, uint8_t *to) {
        asm volatile("" : "+v"(at));       // (keeps it 32 bits)
        __builtin_amdgcn_global_load_lds((global_ptr_t)(from + at), (lds_ptr_t)to, 16, 0, 0);
    };
    auto fetch_a = [&](int buf) {
#pragma unroll
        for (int i = 0; i < LA; ++i) request(ga, oa[i], s_buf + buf * BUF + (i * NW + wave) * 1024);
        ga += kBlock;
    };
    auto fetch_b = [&](int buf, int i) { request(gb, ob[i], s_buf + buf * BUF + BM * kBlock + (i * NG + b_first) * 1024); };
    auto fetch_scales = [&](int to) {
        if (wave * 64 >= BM + BN) return;
        asm volatile("" : "+v"(os));
        __builtin_amdgcn_global_load_lds((global_ptr_t)(gs + os), (lds_ptr_t)(s_scale[to] + wave * 64), 4, 0, 0);
        gs += 4;
    };
    const int wm = wave % WM * (BM / WM), wn = wave / WM * (BN / WN);
    const uint32_t at0 = l31 * kBlock + (half ^ ((l31 >> 1) & 7)) * 16;
    const uint32_t at_a = (uint32_t)(uintptr_t)(lds_ptr_t)&s_buf[0] + wm * kBlock + at0;
    const uint32_t at_b = (uint32_t)(uintptr_t)(lds_ptr_t)&s_buf[0] + (BM + wn) * kBlock + at0;
    const uint32_t lds_scale = (uint32_t)(uintptr_t)(lds_ptr_t)&s_scale[0][0];
    const uint32_t at_sa = lds_scale + 4 * (wm + l31), at_sb = lds_scale + 4 * (BM + wn + l31);
    f32x16_t acc[MI][NI];
    uint32_t sca[MI], scb[NI];
    bool far = false;
    i32x4_t a[MI][2], b[NI][2];
    uint32_t fa = 0, fb = 0;
    auto read_first = [&](int s) {
        const uint32_t from = ((s >> 2) & 1) * ((BM + BN) * 4) + (s & 3);
        fa = at_a + (s & 1) * BUF;
        fb = at_b + (s & 1) * BUF;
        read_step(fa, fa ^ 32u, fb, fb ^ 32u, a, b);
        read_scales(at_sa + from, at_sb + from, sca, scb);
        if (WIDE && __ballot(!in_reach<FA>(sca) || !in_reach<FB>(scb)) && !balance<FA, FB>(sca, scb)) far = true;
    };
    auto multiply = [&](auto between) {
        __builtin_amdgcn_s_setprio(1);
        multiply_step<WIDE, FA, FB, MI, NI>(a, sca, b, scb, acc, between);
        __builtin_amdgcn_s_setprio(0);
    };
    auto all_b = [&](int s) {              // stage s, or the last one again behind it (a branch would cost the sums' registers)
#pragma unroll
        for (int i = 0; i < LB; ++i) fetch_b(s & 1, i);
        if (s + 1 < stages) gb += kBlock;
    };
    const unsigned total = (unsigned)p.ntm * (unsigned)p.ntn * (unsigned)p.splits;
    aim(blockIdx.x, total);
    fetch_scales(0);
    fetch_a(0);
    all_b(0);
    for (unsigned number = blockIdx.x; ; number += gridDim.x) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        if constexpr (PHASES) {
            all_b(1);
            if (number == blockIdx.x) __builtin_amdgcn_s_waitcnt(0x0f70 + LB);  // vmcnt(LB): all but stage 1's
            phase_end();
            if (group == 1) phase_end();
        }
        for (int s = 0; s < stages; ++s) {
            if constexpr (!PHASES) {
                __builtin_amdgcn_s_waitcnt(0x0f70);              // vmcnt(0)
                phase_end();
            }
            if ((s & 3) == 0 && s + 4 < stages) fetch_scales(((s >> 2) + 1) & 1);
            if (s + 1 < stages) fetch_a((s + 1) & 1);
            if (!PHASES && s + 1 < stages) all_b(s + 1);
            read_first(s);
            if constexpr (PHASES) phase_end();
            multiply([](int) {});
            if constexpr (PHASES) phase_end();
            read_step(fa ^ 64u, fa ^ 96u, fb ^ 64u, fb ^ 96u, a, b);
            if constexpr (!PHASES) multiply([](int) {});
            else {
                if (group == 1) __builtin_amdgcn_s_waitcnt(0x0f70);
                phase_end();
                multiply([&](int u) {
                    if (u % 2) return;
                    keep_order();
                    fetch_b(s & 1, u / 2);
                    keep_order();
                });
                if (s + 3 < stages) gb += kBlock;
                if (group == 0) __builtin_amdgcn_s_waitcnt(0x0f70 + LB);
                phase_end();
            }
        }
        if (PHASES && group == 0) phase_end();
        __builtin_amdgcn_s_waitcnt(0x0f70);
        if (WIDE && far) {
            sums_far<FA, FB, 32>(p, m0 + wm, n0 + wn, split * p.kb_split, split * p.kb_split + stages, 1, acc);
            far = false;
        }
        phase_end();
        const int64_t m_out = m0, n_out = n0;
        const int split_out = split;
        const bool more = PHASES && number + gridDim.x < total;
        if (more) {                        // the next tile's first stage
            aim(number + gridDim.x, total);
            fetch_scales(0);
            fetch_a(0);
            all_b(0);
        }
        leave<WIDE, BM, BN, WM, WN>(p, split_out, m_out, n_out, acc, (uint32_t)(uintptr_t)(lds_ptr_t)&s_buf[BUF]);
        if (!more) break;
        phase_end();
    }
}

// The slices' sums, joined in order.
__global__ __launch_bounds__(kThreads) void k_q8_join(const float *__restrict__ part, int splits, int64_t m, int64_t n, MmArgs p)
{
    const int64_t quads = (n + 3) / 4, q = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (q >= m * quads) return;
    const int64_t i = q / quads, j = (q - i * quads) * 4;
    const float *r = part + i * n + j;
    f32x4_t t = {0.f, 0.f, 0.f, 0.f};
    if (j + 4 <= n) {
        auto slice = [&](int s) { return *reinterpret_cast<const f4u_t *>(r + s * m * n); };
        auto add = [&](f4u_t v) { t += f32x4_t{v[0], v[1], v[2], v[3]}; };
        int s = 0;
        for (; s + 4 <= splits; s += 4) {                    // four requested together
            const f4u_t v0 = slice(s), v1 = slice(s + 1), v2 = slice(s + 2), v3 = slice(s + 3);
            add(v0);
            add(v1);
            add(v2);
            add(v3);
        }
        for (; s < splits; ++s) add(slice(s));
    } else {
        for (int s = 0; s < splits; ++s)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j + u < n) t[u] += r[s * m * n + u];
    }
    store4(p, 0, i, j, t);
}

// Products of few rows on one side: every row of the other is read once, and that bounds them.  A wavefront multiplies MI x NI
// tiles of 16 x 16 straight from memory, widened whatever the output (the matrix cores wait here).  KS wavefronts share a tile,
// each with every KS-th block of columns, and join their sums in order through LDS, so that a short table still has enough
// loads under way.
template <int MI, int NI, int KS, int FA, int FB>
__global__ __launch_bounds__(kThreads) void k_q8_direct(MmArgs p)
{
    constexpr int NW = kThreads / 64;
    __shared__ __align__(16) float s_part[KS > 1 ? NW * MI * NI * 256 : 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l15 = lane & 15, kg = lane >> 4, ks = wave % KS;
    const int64_t tile = (int64_t)blockIdx.x * (NW / KS) + wave / KS;
    const int64_t tm = tile % p.ntm, tn = tile / p.ntm;
    const bool in = tn < p.ntn;            // (KS > 1: a workgroup's wavefronts alike, as the grid is exact)
    f32x4_t acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (in) {
        const uint8_t *ra[MI], *sa[MI], *rb[NI], *sb[NI];
        bool far = false;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t r = min((tm * MI + i) * 16 + l15, p.m - 1);
            ra[i] = p.a + r * p.lda;
            sa[i] = p.as + r * p.ldas;
        }
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int64_t r = min((tn * NI + j) * 16 + l15, p.n - 1);
            rb[j] = p.b + r * p.ldb;
            sb[j] = p.bs + r * p.ldbs;
        }
        for (int kb = ks; kb < p.nkb; kb += KS) {
            const int at0 = kb * kBlock + kg * 16, at1 = at0 + 64;
            i32x4_t qa[MI][2], qb[NI][2];
            uint32_t ba[MI], bb[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                qb[j][0] = *reinterpret_cast<const i32x4_t *>(rb[j] + at0);
                qb[j][1] = *reinterpret_cast<const i32x4_t *>(rb[j] + at1);
                bb[j] = sb[j][kb];
            }
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                qa[i][0] = *reinterpret_cast<const i32x4_t *>(ra[i] + at0);
                qa[i][1] = *reinterpret_cast<const i32x4_t *>(ra[i] + at1);
                ba[i] = sa[i][kb];
            }
            if (__ballot(!in_reach<FA>(ba) || !in_reach<FB>(bb)) && !balance<FA, FB>(ba, bb)) far = true;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8_t wb[NI][2];
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int s = 0; s < 2; ++s) wb[j][s] = widen8<FB>(qb[j][h][2 * s], qb[j][h][2 * s + 1], scale_of(bb[j]));
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    bf16x8_t wa[2];
#pragma unroll
                    for (int s = 0; s < 2; ++s) wa[s] = widen8<FA>(qa[i][h][2 * s], qa[i][h][2 * s + 1], scale_of(ba[i]));
#pragma unroll
                    for (int j = 0; j < NI; ++j)
#pragma unroll
                        for (int s = 0; s < 2; ++s) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][s], wa[s], acc[i][j], 0, 0, 0);
                }
            }
        }
        if (far) sums_far<FA, FB, 16>(p, tm * MI * 16, tn * NI * 16, ks, p.nkb, KS, acc);
    }
    if constexpr (KS > 1) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) *reinterpret_cast<f32x4_t *>(s_part + ((wave * MI * NI + i * NI + j) * 64 + lane) * 4) = acc[i][j];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < MI * NI; ++u) {                  // a wavefront joins every KS-th tile
            if (u % KS != ks) continue;
            f32x4_t t = *reinterpret_cast<const f32x4_t *>(s_part + (((wave - ks) * MI * NI + u) * 64 + lane) * 4);
#pragma unroll
            for (int w = 1; w < KS; ++w) t += *reinterpret_cast<const f32x4_t *>(s_part + (((wave - ks + w) * MI * NI + u) * 64 + lane) * 4);
            store4(p, 0, (tm * MI + u / NI) * 16 + l15, (tn * NI + u % NI) * 16 + kg * 4, t);
        }
    } else if (in) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) store4(p, 0, (tm * MI + i) * 16 + l15, (tn * NI + j) * 16 + kg * 4, acc[i][j]);
    }
}

// What a product is cut into: tiles of bm x bn in `splits` slices of the columns, or, for `direct`, tiles of 16 mi x 16 ni whose
// columns `ks` wavefronts share.
struct MmPlan {
    bool direct;
    int bm, bn, mi, ni, ks;
    int64_t ntm, ntn;
    int splits, kb_split;
};
static MmPlan mm_plan(int64_t m, int64_t n, int64_t k, bool wide)
{
    MmPlan t{};
    const int64_t nkb = (k + kBlock - 1) / kBlock, few = m < n ? m : n;
    t.splits = 1;
    t.kb_split = (int)nkb;
    // Tiles of 16 x 16 for tables of up to 4,096 rows, where a workgroup for every 32 would leave compute units idle (16 rows by
    // 300 over 1,024 columns 3.0 us, in 16 x 32 3.5); 16 x 32 above (by 40,000 rows 10.6 us against 12.9).  From 2^18 rows on
    // there are loads enough without sharing the columns, and tiles of 16 x 64 (16 by 4 M over 128 columns 127 us, in shared 16 x 32
    // 179; by 40,000 over 1,024 13.2 against 10.6).  17 to 32 rows: 2 x 2 tiles (32 by 40,000 over 1,024 13.4 us, in 128 x 128 17.8;
    // 33 rows, fp32, in 256 x 128 30).
    if (few <= 32) {
        const int64_t many = m < n ? n : m;
        const int across = few > 16 ? 2 : many >= ((int64_t)1 << 18) ? 4 : many > 4096 ? 2 : 1;
        t.direct = true;
        t.mi = few > 16 ? 2 : m > n ? across : 1;
        t.ni = few > 16 ? 2 : m > n ? 1 : across;
        t.ks = many >= ((int64_t)1 << 18) ? 1 : 4;
        t.ntm = (m + 16 * t.mi - 1) / (16 * t.mi);
        t.ntn = (n + 16 * t.ni - 1) / (16 * t.ni);
        return t;
    }
    // Tiles of 256 x 256 where they fill three quarters of the compute units (14,951 x 1,024 over 8,192 columns, 236 tiles, bf16: 100 us,
    // in 128 x 128 125; 8,192 x 1,024 over 14,976, 128 tiles: 117 and 124, after a rest 171 and 142).  Widened, where the matrix
    // instructions take twice as long, 256 x 128 otherwise, if they do (the same sizes: 256 tiles in 198 us, in 256 x 256 203, in 128 x 128
    // 217; after a rest 191, 260 and 226).  Below, tiles of 128 x 128.
    // The columns are cut into slices of four blocks at least, until there is a workgroup for each compute unit: a second one on it
    // multiplies no faster for what joining costs (2,048 x 2,048 over 2,048 bf16, 256 tiles: 15.2 us, in two slices 26.7).  Joining takes
    // 4 us, as long as eight blocks, so up to 15 blocks stay whole (1,024 x 1,024 over 1,024: 9.5 us, in two slices 14.9; 64 x 2,000
    // over 2,000 fp32, 16 blocks: in four slices 12.5 us, in two 15.7).
    auto tiles_of = [&](int64_t bm, int64_t bn) { return ((m + bm - 1) / bm) * ((n + bn - 1) / bn); };
    t.bm = tiles_of(256, 256) >= 192 || (wide && tiles_of(256, 128) >= 192) ? 256 : 128;
    t.bn = tiles_of(256, 256) >= 192 ? 256 : 128;
    t.ntm = (m + t.bm - 1) / t.bm;
    t.ntn = (n + t.bn - 1) / t.bn;
    const int64_t tiles = t.ntm * t.ntn, most = nkb >= 16 ? nkb / 4 : 1;
    int64_t splits = tiles >= 256 ? 1 : 256 / tiles;
    if (splits > most) splits = most;
    const int64_t each = (((nkb + splits - 1) / splits) + 3) / 4 * 4;
    t.kb_split = (int)each;
    t.splits = (int)((nkb + each - 1) / each);
    return t;
}

size_t q8_matmul_work_bytes(int64_t m, int64_t n, int64_t k)
{
    if (m == 0 || n == 0) return 0;
    const int a = mm_plan(m, n, k, false).splits, b = mm_plan(m, n, k, true).splits, splits = a > b ? a : b;
    return splits > 1 ? ((size_t)splits * (size_t)m * (size_t)n * 4 + 255) / 256 * 256 : 0;
}

template <int FA, int FB>
static void mm_go(stx_ctx *c, const MmPlan &t, bool wide, const MmArgs &p)
{
    if (t.direct) {
        const int per = 4 / t.ks;
        const dim3 grid((unsigned)((t.ntm * t.ntn + per - 1) / per));
        ProfScope prof(c, "k_q8_direct");
#define STX_DIRECT(MI, NI, KS) hipLaunchKernelGGL((k_q8_direct<MI, NI, KS, FA, FB>), grid, dim3(256), 0, c->stream, p)
        if (t.mi == 2 && t.ni == 2 && t.ks == 4) STX_DIRECT(2, 2, 4);
        else if (t.mi == 2 && t.ni == 2) STX_DIRECT(2, 2, 1);
        else if (t.mi == 4) STX_DIRECT(4, 1, 1);
        else if (t.ni == 4) STX_DIRECT(1, 4, 1);
        else if (t.mi == 2) STX_DIRECT(2, 1, 4);
        else if (t.ni == 2) STX_DIRECT(1, 2, 4);
        else STX_DIRECT(1, 1, 4);
#undef STX_DIRECT
        return;
    }
    const int64_t tiles = t.ntm * t.ntn * t.splits;
    const dim3 grid((unsigned)(t.bm == 128 ? tiles : tiles < 256 ? tiles : 256));
    ProfScope prof(c, "k_q8_mm");
    if (t.bm != t.bn) {
        hipLaunchKernelGGL((k_q8_mm<256, 128, 4, 2, true, FA, FB>), grid, dim3(512), 0, c->stream, p);
    } else if (t.bm == 256) {
        if (wide) hipLaunchKernelGGL((k_q8_mm<256, 256, 2, 4, true, FA, FB>), grid, dim3(512), 0, c->stream, p);
        else hipLaunchKernelGGL((k_q8_mm<256, 256, 2, 4, false, FA, FB>), grid, dim3(512), 0, c->stream, p);
    } else {
        if (wide) hipLaunchKernelGGL((k_q8_mm<128, 128, 2, 2, true, FA, FB>), grid, dim3(256), 0, c->stream, p);
        else hipLaunchKernelGGL((k_q8_mm<128, 128, 2, 2, false, FA, FB>), grid, dim3(256), 0, c->stream, p);
    }
}

stx_status launch_q8_matmul(stx_ctx *c, const stx_q8 *a, const stx_q8 *b, int dtype, void *out, int64_t ldo, void *work)
{
    const bool wide = dtype == STX_F32;
    const MmPlan t = mm_plan(a->rows, b->rows, a->cols, wide);
    MmArgs p{a->codes, a->scales, b->codes, b->scales, a->ld, a->ld_scale, b->ld, b->ld_scale, a->rows, b->rows,
             (int)((a->cols + kBlock - 1) / kBlock), t.kb_split, t.splits, (int)t.ntm, (int)t.ntn, out, ldo, dtype, 0};
    // Outputs beyond the caches go past them: 16,384 x 40,448 bf16 over 256 columns in 325 us in place of 423, over 1,024 (40,559)
    // 721 in place of 890.  Rows that are not whole lines leave parts of lines, which meet in the caches only where tiles are short
    // (4,096 x 14,951: over 128 columns 51 us past the caches and 35 through them; over 256, by 16,384 x 40,559, 523 and 550; over 512
    // 62 and 55, after a rest 63 and 66).  fp16 outputs go through them (the first of these 404 us; leave).
    const int64_t size = dtype == STX_F32 ? 4 : 2;
    const bool lines = ldo * size % 128 == 0 && (uintptr_t)out % 128 == 0;
    p.past = t.splits == 1 && p.m * p.n * size >= ((int64_t)64 << 20) && (lines || p.nkb >= 2);
    if (t.splits > 1) {
        p.out = work;
        p.ldo = p.n;
        p.dtype = STX_F32;
    }
    const bool ea = a->format == STX_E4M3, eb = b->format == STX_E4M3;
    if (ea && eb) mm_go<STX_E4M3, STX_E4M3>(c, t, wide, p);
    else if (ea) mm_go<STX_E4M3, STX_E5M2>(c, t, wide, p);
    else if (eb) mm_go<STX_E5M2, STX_E4M3>(c, t, wide, p);
    else mm_go<STX_E5M2, STX_E5M2>(c, t, wide, p);
    if (t.splits > 1) {
        p.out = out;
        p.ldo = ldo;
        p.dtype = dtype;
        ProfScope prof(c, "k_q8_join");
        const int64_t quads = p.m * ((p.n + 3) / 4);
        hipLaunchKernelGGL(k_q8_join, dim3((unsigned)((quads + kThreads - 1) / kThreads)), dim3(kThreads), 0, c->stream, (const float *)work,
                           t.splits, p.m, p.n, p);
    }
    return hip_ok(hipGetLastError());
}

}  // namespace stx
