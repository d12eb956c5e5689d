// Rows in 8 bits, along their own axis and along the other one.
//
// Bound by memory: an element is read once and a code (or two) written for it.  A block's scale needs its largest magnitude
// first, so its elements wait in registers.  Along the rows that is an octet of 16 lanes (stx_fp8.h).  For the transposed
// matrix, whose blocks are 128 rows of one column, a workgroup takes 128 rows of 128 columns: every thread holds 8 rows of an
// octet, so that 8 codes of a column are neighbours in its registers, and the codes turn in LDS.
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
    float v[8];
    octet_floats(request_octet(x + row * ld, blk, l16, cols), blk, l16, cols, v);
    store_q8_octet<T, FORMAT>(q, row, blk, l16, v);
}

constexpr int kTurnPitch = kBlock + 8;     // bytes of a column's codes in LDS

// A thread's 8 x 8 elements: rows 8 (thread / 16) + i, columns of its octet.
template <class T, int FORMAT, int FORMAT_T>
__global__ __launch_bounds__(kThreads) void k_q8_turn(const T *__restrict__ x, int64_t rows, int64_t cols, int64_t ld, int col_blocks, Q8Out q, Q8Out qt)
{
    __shared__ uint32_t s_most[4][kBlock];
    __shared__ __align__(16) uint8_t s_codes[kBlock * kTurnPitch];
    const int l16 = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const int row_blk = (int)(blockIdx.x / (unsigned)col_blocks), blk = (int)(blockIdx.x % (unsigned)col_blocks);
    const int64_t row0 = (int64_t)row_blk * kBlock + rg * 8;
    Octet<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) raw[i] = request_octet(x + (row0 + i) * ld, blk, l16, row0 + i < rows ? cols : 0);
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) octet_floats(raw[i], blk, l16, row0 + i < rows ? cols : 0, v[i]);
    if (q.codes) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (row0 + i < rows) store_q8_octet<T, FORMAT>(q, row0 + i, blk, l16, v[i]);
    }
    uint32_t most[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        most[j] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) most[j] = max(most[j], finite_bits(v[i][j]));
        most[j] = max(most[j], (uint32_t)__shfl_xor((int)most[j], 16, 64));
        most[j] = max(most[j], (uint32_t)__shfl_xor((int)most[j], 32, 64));
        if ((threadIdx.x & 48) == 0) s_most[wave][octet_pos<T>(0, l16, j)] = most[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = octet_pos<T>(0, l16, j);
        const uint32_t byte = block_scale<FORMAT_T>(max(max(s_most[0][c], s_most[1][c]), max(s_most[2][c], s_most[3][c])));
        const float down = scale_down(byte);
        float s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = scaled<FORMAT_T>(v[i][j], down);
        *reinterpret_cast<uint2 *>(s_codes + c * kTurnPitch + rg * 8) =
            make_uint2(pack4<FORMAT_T>(s[0], s[1], s[2], s[3]), pack4<FORMAT_T>(s[4], s[5], s[6], s[7]));
        const int64_t col = (int64_t)blk * kBlock + c;
        if (rg == 0 && col < cols) qt.scales[col * qt.ld_scale + row_blk] = (uint8_t)byte;
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {          // 16 bytes a thread, a column's 128 in 8 threads
        const int c = u * 32 + (threadIdx.x >> 3), at = (threadIdx.x & 7) * 16;
        const int64_t col = (int64_t)blk * kBlock + c;
        if (col < cols) {
            const uint2 a = *reinterpret_cast<const uint2 *>(s_codes + c * kTurnPitch + at);
            const uint2 b = *reinterpret_cast<const uint2 *>(s_codes + c * kTurnPitch + at + 8);
            *reinterpret_cast<uint4 *>(qt.codes + col * qt.ld + (int64_t)row_blk * kBlock + at) = make_uint4(a.x, a.y, b.x, b.y);
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
        ProfScope prof(c, "k_q8_rows");
        const dim3 grid((unsigned)((rows * cb + kThreads / 16 - 1) / (kThreads / 16)));
        if (q->format == STX_E4M3) hipLaunchKernelGGL((k_q8_rows<T, STX_E4M3>), grid, dim3(kThreads), 0, c->stream, xt, rows, cols, ld, (int)cb, out_of(q));
        else hipLaunchKernelGGL((k_q8_rows<T, STX_E5M2>), grid, dim3(kThreads), 0, c->stream, xt, rows, cols, ld, (int)cb, out_of(q));
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
