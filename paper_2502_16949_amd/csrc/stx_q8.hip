// Rows in 8 bits, along their own axis and along the other one.
//
// Bound by memory: an element is read once and a code (or two) written for it.  A block's scale needs its largest magnitude
// first, so its elements wait in registers.  Along the rows that is an octet of 16 lanes (stx_fp8.h).  For the transposed
// matrix, whose blocks are 128 rows of one column, a workgroup takes 128 rows of 128 columns: every thread holds 8 rows of an
// octet, so that 8 codes of a column are neighbours in its registers, and the codes turn in LDS.  16-bit numbers stay in pairs from
// memory to their codes; as floats they took four times the arithmetic (8,192 x 1,024 bf16 turned: 12.6 us, so 10.4).
#include "stx_device.h"
#include "stx_ops.h"

namespace stx {

template <class T, int FORMAT>
__global__ __launch_bounds__(kThreads) void k_q8_rows(const T *__restrict__ x, int64_t rows, int64_t cols, int64_t ld, int blocks, Q8Out q)
{
    const int l16 = threadIdx.x & 15;
    const int64_t i = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);     // blocks of all rows, end to end
    const int64_t row = i / blocks;
    if (row >= rows) return;
    const int blk = (int)(i - row * blocks);
    Octet<T> o = request_octet(x + row * ld, blk, l16, cols);
    settle_octet(o, blk, l16, cols);
    store_q8_octet<T, FORMAT>(q, row, blk, l16, o);
}

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
constexpr int kTurnPitch = kBlock + 8;     // bytes of a column's codes in LDS
// Every die takes a run of consecutive blocks (workgroups go round the dies in turn), along stripes of 8 blocks of rows, so that the
// scales of neighbours, single bytes both ways, meet in its L2 (8,192 x 14,951 bf16 both ways in 125 us in order, so in 119; 114 with
// the transposed codes, whole lines, past the caches; now 109).
constexpr unsigned kDies = 8, kTurnStripe = 8;

// Element j of eight octets: the largest finite magnitude (bits of an fp32), for all j, and the codes.
template <class T>
__device__ inline void column_largest(const Octet<T> (&o)[8], uint32_t (&most)[8])
{
#pragma unroll
    for (int k = 0; k < (int)sizeof(T) * 2; ++k) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = o[i].w[k];
        if constexpr (sizeof(T) == 4) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, w[i]);
            most[k] = largest<8>(v);
        } else {
            largest_pair<T, 8>(w, most[2 * k], most[2 * k + 1]);
        }
    }
}
template <class T, int FORMAT>
__device__ inline uint2 column_codes(const Octet<T> (&o)[8], int j, float scale)
{
    uint32_t c[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (sizeof(T) == 4) {
            c[h] = code4<FORMAT>(__builtin_bit_cast(float, o[4 * h].w[j]), __builtin_bit_cast(float, o[4 * h + 1].w[j]),
                                 __builtin_bit_cast(float, o[4 * h + 2].w[j]), __builtin_bit_cast(float, o[4 * h + 3].w[j]), scale);
        } else {
            const uint32_t take = j & 1 ? 0x07060302u : 0x05040100u;            // the same half of two words
            c[h] = code4<T, FORMAT>(__builtin_amdgcn_perm(o[4 * h + 1].w[j / 2], o[4 * h].w[j / 2], take),
                                    __builtin_amdgcn_perm(o[4 * h + 3].w[j / 2], o[4 * h + 2].w[j / 2], take), scale);
        }
    }
    return make_uint2(c[0], c[1]);
}

// A thread's 8 x 8 elements: rows 8 (thread / 16) + i, columns of its octet.
template <class T, int FORMAT, int FORMAT_T>
__global__ __launch_bounds__(kThreads) void k_q8_turn(const T *__restrict__ x, int64_t rows, int64_t cols, int64_t ld, int col_blocks, Q8Out q, Q8Out qt)
{
    __shared__ uint32_t s_most[4][kBlock];
    __shared__ __align__(16) uint8_t s_codes[kBlock * kTurnPitch];
    const int l16 = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const unsigned row_blocks = gridDim.x / (unsigned)col_blocks, die = blockIdx.x % kDies, each = gridDim.x / kDies, more = gridDim.x % kDies;
    const unsigned number = die * each + (die < more ? die : more) + blockIdx.x / kDies, stripe = kTurnStripe * (unsigned)col_blocks;
    const unsigned first = number / stripe * kTurnStripe, high = min(kTurnStripe, row_blocks - first), in = number % stripe;
    const int row_blk = (int)(first + in % high), blk = (int)(in / high);
    const int64_t row0 = (int64_t)row_blk * kBlock + rg * 8;
    Octet<T> o[8];                         // rows behind the last one: its own, made 0 below
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = request_octet(x + min(row0 + i, rows - 1) * ld, blk, l16, cols);
#pragma unroll
    for (int i = 0; i < 8; ++i) settle_octet(o[i], blk, l16, cols);
    if (row0 + 8 > rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int k = 0; k < (int)sizeof(T) * 2; ++k) o[i].w[k] = row0 + i < rows ? o[i].w[k] : 0u;
    }
    if (q.codes) {
        uint32_t byte[8];                  // (written together, these and the other way's below: beside the codes 8,192 x 14,951 bf16 took 114 us, so 109)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            byte[i] = block_scale<FORMAT>(row16_max(largest(o[i])));
            if (row0 + i < rows) store_codes<T>(q, row0 + i, blk, l16, code8<T, FORMAT>(o[i], scale_of(byte[i])));
        }
        if (l16 == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (row0 + i < rows) q.scales[(row0 + i) * q.ld_scale + blk] = (uint8_t)byte[i];
        }
    }
    uint32_t most[8];
    column_largest(o, most);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        most[j] = max(most[j], (uint32_t)__shfl_xor((int)most[j], 16, 64));
        most[j] = max(most[j], (uint32_t)__shfl_xor((int)most[j], 32, 64));
        if ((threadIdx.x & 48) == 0) s_most[wave][octet_pos<T>(0, l16, j)] = most[j];
    }
    __syncthreads();
    uint32_t byte_t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = octet_pos<T>(0, l16, j);
        byte_t[j] = block_scale<FORMAT_T>(max(max(s_most[0][c], s_most[1][c]), max(s_most[2][c], s_most[3][c])));
        *reinterpret_cast<uint2 *>(s_codes + c * kTurnPitch + rg * 8) = column_codes<T, FORMAT_T>(o, j, scale_of(byte_t[j]));
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {          // 16 bytes a thread, a column's 128 in 8 threads: whole lines, past the caches
        const int c = u * 32 + (threadIdx.x >> 3), at = (threadIdx.x & 7) * 16;
        const int64_t col = (int64_t)blk * kBlock + c;
        if (col < cols) {
            const uint2 a = *reinterpret_cast<const uint2 *>(s_codes + c * kTurnPitch + at);
            const uint2 b = *reinterpret_cast<const uint2 *>(s_codes + c * kTurnPitch + at + 8);
            __builtin_nontemporal_store(u32x4_t{a.x, a.y, b.x, b.y}, reinterpret_cast<u32x4_t *>(qt.codes + col * qt.ld + (int64_t)row_blk * kBlock + at));
        }
    }
    if (rg == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t col = (int64_t)blk * kBlock + octet_pos<T>(0, l16, j);
            if (col < cols) qt.scales[col * qt.ld_scale + row_blk] = (uint8_t)byte_t[j];
        }
    }
}

static Q8Out out_of(const stx_q8 *q) { return q ? Q8Out{q->codes, q->scales, q->ld, q->ld_scale} : Q8Out{}; }

template <class T>
static void quantize_go(stx_ctx *c, int64_t rows, int64_t cols, int64_t ld, const void *x, const stx_q8 *q, const stx_q8 *qt)
{
    const int64_t cb = (cols + kBlock - 1) / kBlock, rb = (rows + kBlock - 1) / kBlock;
    const T *xt = (const T *)x;
    if (!qt) {
        const int64_t most = kMaxItems / kThreads * (kThreads / 16) / cb;       // rows of one launch
        Q8Out to = out_of(q);
        for (int64_t left = rows; left > 0; left -= most, xt += most * ld, to.codes += most * to.ld, to.scales += most * to.ld_scale) {
            const int64_t now = left < most ? left : most;
            ProfScope prof(c, "k_q8_rows");
            const dim3 grid((unsigned)((now * cb + kThreads / 16 - 1) / (kThreads / 16)));
            if (q->format == STX_E4M3) hipLaunchKernelGGL((k_q8_rows<T, STX_E4M3>), grid, dim3(kThreads), 0, c->stream, xt, now, cols, ld, (int)cb, to);
            else hipLaunchKernelGGL((k_q8_rows<T, STX_E5M2>), grid, dim3(kThreads), 0, c->stream, xt, now, cols, ld, (int)cb, to);
        }
        return;
    }
    ProfScope prof(c, "k_q8_turn");
    const dim3 grid((unsigned)(rb * cb));
    const bool e4 = !q || q->format == STX_E4M3, e4t = qt->format == STX_E4M3;
#define STX_TURN(F, FT) \
    hipLaunchKernelGGL((k_q8_turn<T, F, FT>), grid, dim3(kThreads), 0, c->stream, xt, rows, cols, ld, (int)cb, out_of(q), out_of(qt))
    if (e4 && e4t) STX_TURN(STX_E4M3, STX_E4M3);
    else if (e4) STX_TURN(STX_E4M3, STX_E5M2);
    else if (e4t) STX_TURN(STX_E5M2, STX_E4M3);
    else STX_TURN(STX_E5M2, STX_E5M2);
#undef STX_TURN
}

stx_status launch_q8_quantize(stx_ctx *c, int dtype, int64_t rows, int64_t cols, int64_t ld, const void *x, const stx_q8 *q,
                              const stx_q8 *qt)
{
    if (dtype == STX_F32) quantize_go<float>(c, rows, cols, ld, x, q, qt);
    else if (dtype == STX_BF16) quantize_go<bf16_t>(c, rows, cols, ld, x, q, qt);
    else quantize_go<f16_t>(c, rows, cols, ld, x, q, qt);
    return hip_ok(hipGetLastError());
}

}  // namespace stx
