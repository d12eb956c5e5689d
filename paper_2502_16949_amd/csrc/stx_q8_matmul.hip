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
//   front of v_mfma_f32_16x16x32_bf16, whose products are whole: 1e-7 of the result, at half the rate.
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
};

// One fragment of an operand: 32 codes a lane, of row lane % 16.  Which columns a lane holds does not matter to a sum as long as
// both operands agree.
template <int FORMAT>
__device__ inline bf16x2_t widen2(int w, float scale, bool hi)
{
    if constexpr (FORMAT == STX_E4M3) return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    else return hi ? __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, false);
}
template <int FORMAT>
__device__ inline bf16x8_t widen8(int lo, int hi, float scale)
{
    const bf16x2_t a = widen2<FORMAT>(lo, scale, false), b = widen2<FORMAT>(lo, scale, true);
    const bf16x2_t c = widen2<FORMAT>(hi, scale, false), d = widen2<FORMAT>(hi, scale, true);
    return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A piece is what one pass over a step takes of a row: all 32 codes of a lane, or, widened, half of them at a time (registers).
template <bool WIDE> struct Piece;
template <> struct Piece<false> {
    i32x4_t lo, hi;
    __device__ void load(const uint8_t *row, int at0, int at1, int)
    {
        lo = *reinterpret_cast<const i32x4_t *>(row + at0);
        hi = *reinterpret_cast<const i32x4_t *>(row + at1);
    }
};
template <> struct Piece<true> {
    i32x4_t lo;
    __device__ void load(const uint8_t *row, int at0, int at1, int half) { lo = *reinterpret_cast<const i32x4_t *>(row + (half ? at1 : at0)); }
};
template <bool WIDE, int FORMAT> struct Frag;
template <int FORMAT> struct Frag<false, FORMAT> {
    i32x8_t v;
    int scale;
    __device__ void set(const Piece<false> &p, uint32_t byte)
    {
        v = i32x8_t{p.lo[0], p.lo[1], p.lo[2], p.lo[3], p.hi[0], p.hi[1], p.hi[2], p.hi[3]};
        scale = (int)byte;
    }
};
template <int FORMAT> struct Frag<true, FORMAT> {
    bf16x8_t v[2];
    __device__ void set(const Piece<true> &p, uint32_t byte)
    {
        const float s = __builtin_bit_cast(float, byte << 23);
        v[0] = widen8<FORMAT>(p.lo[0], p.lo[1], s);
        v[1] = widen8<FORMAT>(p.lo[2], p.lo[3], s);
    }
};
// acc += B A^T: a lane has row lane % 16 of A and 4 consecutive rows of B.
template <int FA, int FB>
__device__ inline f32x4_t multiply(const Frag<false, FB> &b, const Frag<false, FA> &a, f32x4_t acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, acc, FB, FA, 0, b.scale, 0, a.scale);
}
template <int FA, int FB>
__device__ inline f32x4_t multiply(const Frag<true, FB> &b, const Frag<true, FA> &a, f32x4_t acc)
{
#pragma unroll
    for (int s = 0; s < 2; ++s) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[s], a.v[s], acc, 0, 0, 0);
    return acc;
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

// The workgroup's tile: every die takes a run of consecutive tiles (workgroups go round the dies in turn), along stripes of
// kStripe tiles of A, so that what a die reads at a time fits its L2.
constexpr int kDies = 8, kStripe = 8;
__device__ inline void tile_of(const MmArgs &p, int &tm, int &tn, int &split)
{
    const unsigned total = gridDim.x, die = blockIdx.x % kDies, each = total / kDies, more = total % kDies;
    const unsigned i = die * each + (die < more ? die : more) + blockIdx.x / kDies;
    const unsigned tiles = (unsigned)p.ntm * (unsigned)p.ntn;
    split = (int)(i / tiles);
    const unsigned t = i % tiles, stripe = t / (unsigned)(kStripe * p.ntn), r = t % (unsigned)(kStripe * p.ntn);
    const unsigned first = stripe * kStripe, high = min((unsigned)kStripe, (unsigned)p.ntm - first);
    tm = (int)(first + r % high);
    tn = (int)(r / high);
}

typedef const __attribute__((address_space(1))) void *global_ptr_t;
typedef __attribute__((address_space(3))) void *lds_ptr_t;

// A BM x BN tile by WM x WN wavefronts.  A step is one block of 128 columns: its codes go straight to LDS, a row's 128 bytes
// in a line whose 16-byte pieces are permuted by the row (piece c of row r at c ^ (r / 2 % 8)), and a lane reads
// pieces g and g + 4 of its row, g = lane / 16: 2.88 ns a read and CU, as 64 lanes side by side; pieces 2 g and 2 g + 1 3.65.  Two buffers: a step's loads are under way while the one before it is computed.
template <int BM, int BN, int WM, int WN, bool WIDE, int FA, int FB>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_q8_mm(MmArgs p)
{
    constexpr int NW = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16, LA = BM / 8 / NW, LB = BN / 8 / NW;
    static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "whole rounds of loads");
    __shared__ __align__(16) uint8_t s_a0[BM * kBlock], s_a1[BM * kBlock], s_b0[BN * kBlock], s_b1[BN * kBlock];
    __shared__ uint32_t s_scale[2][BM + BN];
    int tm, tn, split;
    tile_of(p, tm, tn, split);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int l15 = lane & 15, kg = lane >> 4;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int kb0 = split * p.kb_split, kb1 = min(kb0 + p.kb_split, p.nkb);
    // loads: a wavefront's 64 pieces are 8 rows; rows behind the last one repeat it
    static_assert(NW % 2 == 0, "a wavefront's rows begin at the same place of 16 in every round");
    const int piece = ((lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7)) * 16;
    uint32_t oa[LA], ob[LB];
#pragma unroll
    for (int i = 0; i < LA; ++i) oa[i] = (uint32_t)(min((int64_t)((i * NW + wave) * 8 + (lane >> 3)), p.m - 1 - m0) * p.lda) + piece;
#pragma unroll
    for (int i = 0; i < LB; ++i) ob[i] = (uint32_t)(min((int64_t)((i * NW + wave) * 8 + (lane >> 3)), p.n - 1 - n0) * p.ldb) + piece;
    const uint8_t *ga = p.a + m0 * p.lda + (int64_t)kb0 * kBlock, *gb = p.b + n0 * p.ldb + (int64_t)kb0 * kBlock;
    auto fetch = [&](uint8_t *sa, uint8_t *sb) {
#pragma unroll
        for (int i = 0; i < LA; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr_t)(ga + oa[i]), (lds_ptr_t)(sa + (i * NW + wave) * 1024), 16, 0, 0);
#pragma unroll
        for (int i = 0; i < LB; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr_t)(gb + ob[i]), (lds_ptr_t)(sb + (i * NW + wave) * 1024), 16, 0, 0);
        ga += kBlock;
        gb += kBlock;
    };
    // scales: a thread brings those of one row, a word for four steps, one group of steps ahead
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    static_assert(BM + BN == NW * 64, "a thread for each row's scales");
    const uint8_t *scales = threadIdx.x < BM ? p.as + min(m0 + (int)threadIdx.x, p.m - 1) * p.ldas
                                             : p.bs + min(n0 + (int)threadIdx.x - BM, p.n - 1) * p.ldbs;
    uint32_t word = *reinterpret_cast<const uint32_t *>(scales + kb0);
    s_scale[(kb0 >> 2) & 1][threadIdx.x] = word;
    f32x4_t acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int at0 = l15 * kBlock + (kg ^ (l15 >> 1)) * 16, at1 = l15 * kBlock + ((kg + 4) ^ (l15 >> 1)) * 16;
    auto compute = [&](const uint8_t *sa, const uint8_t *sb, int kb) {
        const uint8_t *sc = reinterpret_cast<const uint8_t *>(s_scale[(kb >> 2) & 1]) + (kb & 3);
        uint32_t scb[NI], sca[MI];
#pragma unroll
        for (int j = 0; j < NI; ++j) scb[j] = sc[4 * (BM + wn + j * 16 + l15)];
#pragma unroll
        for (int i = 0; i < MI; ++i) sca[i] = sc[4 * (wm + i * 16 + l15)];
#pragma unroll
        for (int half = 0; half < (WIDE ? 2 : 1); ++half) {
            Frag<WIDE, FB> fb[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                Piece<WIDE> q;
                q.load(sb + (wn + j * 16) * kBlock, at0, at1, half);
                fb[j].set(q, scb[j]);
            }
            Piece<WIDE> next;
            next.load(sa + wm * kBlock, at0, at1, half);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                Frag<WIDE, FA> fa;
                fa.set(next, sca[i]);
                if (i + 1 < MI) next.load(sa + (wm + (i + 1) * 16) * kBlock, at0, at1, half);
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = multiply<FA, FB>(fb[j], fa, acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);           // no fragments of later rows ahead of these: registers
            }
        }
    };
    // the next group's scales: fetched in its first step, in LDS two steps later (read by nobody since the group before)
    auto scales_ahead = [&](int kb) {
        if ((kb & 3) == 0 && kb + 4 < kb1) word = *reinterpret_cast<const uint32_t *>(scales + kb + 4);
        if ((kb & 3) == 2) s_scale[((kb >> 2) + 1) & 1][threadIdx.x] = word;
    };
    auto arrive = [&]() {                  // this step's loads have come, and every wavefront is done with the other buffer
        __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0)
        __syncthreads();
    };
    fetch(s_a0, s_b0);
    for (int kb = kb0; kb < kb1; kb += 2) {
        arrive();
        if (kb + 1 < kb1) fetch(s_a1, s_b1);
        scales_ahead(kb);
        compute(s_a0, s_b0, kb);
        if (kb + 1 < kb1) {                // (not a break: the accumulators stay where they are)
            arrive();
            if (kb + 2 < kb1) fetch(s_a0, s_b0);
            compute(s_a1, s_b1, kb + 1);
        }
    }
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) store4(p, split, m0 + wm + i * 16 + l15, n0 + wn + j * 16 + kg * 4, acc[i][j]);
}

// The slices' sums, joined in order.
__global__ __launch_bounds__(kThreads) void k_q8_join(const float *__restrict__ part, int splits, int64_t m, int64_t n, MmArgs p)
{
    const int64_t quads = (n + 3) / 4, q = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (q >= m * quads) return;
    const int64_t i = q / quads, j = (q - i * quads) * 4;
    f32x4_t t = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) {
        const float *r = part + ((int64_t)s * m + i) * n + j;
        if (j + 4 <= n) {
            const f4u_t v = *reinterpret_cast<const f4u_t *>(r);
            t += f32x4_t{v[0], v[1], v[2], v[3]};
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j + u < n) t[u] += r[u];
        }
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
            Piece<false> qa[MI], qb[NI];
            uint32_t ba[MI], bb[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) { qb[j].load(rb[j], at0, at1, 0); bb[j] = sb[j][kb]; }
#pragma unroll
            for (int i = 0; i < MI; ++i) { qa[i].load(ra[i], at0, at1, 0); ba[i] = sa[i][kb]; }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                Frag<true, FB> fb[NI];
#pragma unroll
                for (int j = 0; j < NI; ++j) fb[j].set(Piece<true>{half ? qb[j].hi : qb[j].lo}, bb[j]);
#pragma unroll
                for (int i = 0; i < MI; ++i) {
                    Frag<true, FA> fa;
                    fa.set(Piece<true>{half ? qa[i].hi : qa[i].lo}, ba[i]);
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] = multiply<FA, FB>(fb[j], fa, acc[i][j]);
                }
            }
        }
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
static MmPlan mm_plan(int64_t m, int64_t n, int64_t k)
{
    MmPlan t{};
    const int64_t nkb = (k + kBlock - 1) / kBlock, few = m < n ? m : n;
    t.splits = 1;
    t.kb_split = (int)nkb;
    // Tiles of 16 x 16 for tables of up to 4,096 rows, where a workgroup for every 32 would leave compute units idle (16 rows by
    // 300 over 1,024 columns 3.0 us, in 16 x 32 3.5); 16 x 32 above (by 40,000 rows 10.6 us against 12.9).  From 2^18 rows on
    // there are loads enough without sharing the columns, and tiles of 16 x 64 (16 by 4 M over 128 columns 146 us, in shared 16 x 32
    // 179; by 40,000 over 1,024 13.2 against 10.6).  17 to 32 rows: 2 x 2 tiles (32 by 40,000 over 1,024 13.4 us, in 128 x 128 17.8).
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
    const int64_t big = ((m + 255) / 256) * ((n + 255) / 256);
    t.bm = t.bn = big >= 192 ? 256 : 128;
    t.ntm = (m + t.bm - 1) / t.bm;
    t.ntn = (n + t.bn - 1) / t.bn;
    const int64_t tiles = t.ntm * t.ntn, room = t.bm == 256 ? 256 : 512;
    int64_t splits = tiles >= room ? 1 : room / tiles;
    const int64_t most = nkb / 8 > 0 ? nkb / 8 : 1;          // eight blocks a slice at least
    if (splits > most) splits = most;
    const int64_t each = (((nkb + splits - 1) / splits) + 3) / 4 * 4;
    t.kb_split = (int)each;
    t.splits = (int)((nkb + each - 1) / each);
    return t;
}

size_t q8_matmul_work_bytes(int64_t m, int64_t n, int64_t k)
{
    if (m == 0 || n == 0) return 0;
    const MmPlan t = mm_plan(m, n, k);
    return t.splits > 1 ? ((size_t)t.splits * (size_t)m * (size_t)n * 4 + 255) / 256 * 256 : 0;
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
    const dim3 grid((unsigned)(t.ntm * t.ntn * t.splits));
    ProfScope prof(c, "k_q8_mm");
    if (t.bm == 256) {
        if (wide) hipLaunchKernelGGL((k_q8_mm<256, 256, 2, 4, true, FA, FB>), grid, dim3(512), 0, c->stream, p);
        else hipLaunchKernelGGL((k_q8_mm<256, 256, 2, 4, false, FA, FB>), grid, dim3(512), 0, c->stream, p);
    } else {
        if (wide) hipLaunchKernelGGL((k_q8_mm<128, 128, 2, 2, true, FA, FB>), grid, dim3(256), 0, c->stream, p);
        else hipLaunchKernelGGL((k_q8_mm<128, 128, 2, 2, false, FA, FB>), grid, dim3(256), 0, c->stream, p);
    }
}

stx_status launch_q8_matmul(stx_ctx *c, const stx_q8 *a, const stx_q8 *b, int dtype, void *out, int64_t ldo, void *work)
{
    const MmPlan t = mm_plan(a->rows, b->rows, a->cols);
    MmArgs p{a->codes, a->scales, b->codes, b->scales, a->ld, a->ld_scale, b->ld, b->ld_scale, a->rows, b->rows,
             (int)((a->cols + kBlock - 1) / kBlock), t.kb_split, t.splits, (int)t.ntm, (int)t.ntn, out, ldo, dtype};
    if (t.splits > 1) {
        p.out = work;
        p.ldo = p.n;
        p.dtype = STX_F32;
    }
    const bool wide = dtype == STX_F32, ea = a->format == STX_E4M3, eb = b->format == STX_E4M3;
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
