// Root-mean-square norm of rows with the residual's addition, its 8-bit output, and its backward pass.
//
//   s = x + residual (rounded to the rows' type);  y = s rstd w,  rstd = (mean(s^2) + eps)^-1/2
//   a = dy w;  dx = rstd (a - s rstd^2 mean(a s)) + dsum;  dw = sum_rows dy s rstd
//
// Both directions are bound by memory: a row is read once, held in registers as floats while its sum is formed, and written
// once.  G threads share a row, in octets (stx_fp8.h): the fewest that hold it with up to 32 elements each, a wavefront where
// that suffices, so that up to 2,048 columns the sum needs no barrier.
#include "stx_device.h"
#include "stx_fp8.h"
#include "stx_internal.h"
#include "stx_ops.h"

namespace stx {

// Sum over the G threads that share a row; every one receives it.  G = 256: the whole workgroup, through s_red[slot], where
// calls in turn take slots in turn.
template <int G>
__device__ inline float row_sum(float v, float (*s_red)[4], int slot)
{
    if constexpr (G <= 64) return group_sum<G>(v);
    v = group_sum<64>(v);
    if ((threadIdx.x & 63) == 0) s_red[slot][threadIdx.x >> 6] = v;
    __syncthreads();
    return (s_red[slot][0] + s_red[slot][1]) + (s_red[slot][2] + s_red[slot][3]);
}

template <class T, int G, int ITERS>
__global__ __launch_bounds__(kThreads) void k_rmsnorm(NormArgs a)
{
    constexpr int GROUPS = kThreads / G;
    __shared__ float s_red[1][4];
    const int g = threadIdx.x % G, l16 = g & 15;
    const int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
    if (row >= a.rows) return;             // (G = 256: the whole workgroup)
    const int64_t at = row * a.ld;
    const T *x = (const T *)a.x + at, *res = a.residual ? (const T *)a.residual + at : nullptr;
    T *sum = a.sum ? (T *)a.sum + at : nullptr;
    float s[ITERS][8], r[ITERS][8], ss = 0.f;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) load_octet<T>(x, (it * G + g) >> 4, l16, a.cols, s[it]);
    if (res) {
#pragma unroll
        for (int it = 0; it < ITERS; ++it) load_octet<T>(res, (it * G + g) >> 4, l16, a.cols, r[it]);
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[it][j] += r[it][j];
    }
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        round_store_octet<T>(sum, (it * G + g) >> 4, l16, a.cols, s[it]);
#pragma unroll
        for (int j = 0; j < 8; ++j) ss += s[it][j] * s[it][j];
    }
    if (!a.y && !a.q.codes && !a.rstd) return;
    const float rstd = 1.0f / sqrtf(row_sum<G>(ss, s_red, 0) / (float)a.cols + a.eps);
    if (g == 0 && a.rstd) a.rstd[row] = rstd;
    if (!a.y && !a.q.codes) return;
    const int blocks = (int)((a.cols + kBlock - 1) / kBlock);
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int blk = (it * G + g) >> 4;
        if (blk >= blocks) break;          // (the 16 lanes of a block leave together)
        float w[8];
        if (a.weight) load_octet_as<T>(a.weight, blk, l16, a.cols, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s[it][j] *= rstd;
            if (a.weight) s[it][j] *= w[j];
        }
        if (a.q.codes) {
            if (a.format == STX_E4M3) store_q8_octet<T, STX_E4M3>(a.q, row, blk, l16, s[it]);
            else store_q8_octet<T, STX_E5M2>(a.q, row, blk, l16, s[it]);
        }
        if (a.y) round_store_octet<T>((T *)a.y + at, blk, l16, a.cols, s[it]);
    }
}

// A workgroup takes rows in turn and keeps its part of dweight in registers; the parts are joined by k_norm_dweight.
template <class T, int G, int ITERS>
__global__ __launch_bounds__(kThreads) void k_rmsnorm_bwd(NormBwdArgs a)
{
    constexpr int GROUPS = kThreads / G;
    __shared__ float s_red[2][4];
    __shared__ float s_dw[GROUPS > 1 ? GROUPS * G * 8 : 1];
    const int g = threadIdx.x % G, grp = threadIdx.x / G, l16 = g & 15;
    float w[ITERS][8], dw[ITERS][8];
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        if (a.weight) load_octet_as<T>(a.weight, (it * G + g) >> 4, l16, a.cols, w[it]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (!a.weight) w[it][j] = 1.f;
            dw[it][j] = 0.f;
        }
    }
    int slot = 0;
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + grp; row < a.rows; row += (int64_t)gridDim.x * GROUPS, slot ^= 1) {
        const int64_t at = row * a.ld;
        float s[ITERS][8], d[ITERS][8], e[ITERS][8];
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            load_octet<T>((const T *)a.sum + at, (it * G + g) >> 4, l16, a.cols, s[it]);
            load_octet<T>((const T *)a.dy + at, (it * G + g) >> 4, l16, a.cols, d[it]);
        }
        if (a.dsum) {
#pragma unroll
            for (int it = 0; it < ITERS; ++it) load_octet<T>((const T *)a.dsum + at, (it * G + g) >> 4, l16, a.cols, e[it]);
        }
        const float rstd = a.rstd[row];
        float dot = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dw[it][j] += d[it][j] * (s[it][j] * rstd);
                d[it][j] *= w[it][j];
                dot += d[it][j] * s[it][j];
            }
        const float c = row_sum<G>(dot, s_red, slot) / (float)a.cols * rstd * rstd;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                d[it][j] = (d[it][j] - s[it][j] * c) * rstd;
                if (a.dsum) d[it][j] += e[it][j];
            }
            round_store_octet<T>((T *)a.dx + at, (it * G + g) >> 4, l16, a.cols, d[it]);
        }
    }
    if (!a.partials) return;
    float *out = a.partials + (int64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        if constexpr (GROUPS > 1) {        // the groups' parts in order
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) s_dw[(grp * 8 + j) * G + g] = dw[it][j];
            __syncthreads();
            if (grp == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float t = s_dw[j * G + g];
#pragma unroll
                    for (int u = 1; u < GROUPS; ++u) t += s_dw[(u * 8 + j) * G + g];
                    dw[it][j] = t;
                }
            }
        }
        if (grp == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t col = octet_pos<T>((it * G + g) >> 4, l16, j);
                if (col < a.cols) out[col] = dw[it][j];
            }
        }
    }
}

// dweight = the workgroups' parts, 16 slices of them side by side and then in order.
__global__ __launch_bounds__(kThreads) void k_norm_dweight(const float *__restrict__ partials, int n, int64_t cols, float *__restrict__ dweight)
{
    __shared__ float s_part[16][17];
    const int c = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int64_t col = (int64_t)blockIdx.x * 16 + c;
    float t = 0.f;
    if (col < cols) {
#pragma unroll 4
        for (int i = slice; i < n; i += 16) t += partials[(int64_t)i * cols + col];
    }
    s_part[slice][c] = t;
    __syncthreads();
    if (slice == 0 && col < cols) {
#pragma unroll
        for (int u = 1; u < 16; ++u) t += s_part[u][c];
        dweight[col] = t;
    }
}

static int row_threads(int64_t cols) { return cols <= 128 ? 16 : cols <= 256 ? 32 : cols <= 2048 ? 64 : 256; }

// Workgroups of a backward pass: four a CU, so that each sums many rows into its part.
static int bwd_blocks(int64_t rows, int64_t cols)
{
    const int64_t groups = kThreads / row_threads(cols), need = (rows + groups - 1) / groups;
    return (int)(need < 1024 ? need : 1024);
}
size_t norm_bwd_work_bytes(int64_t rows, int64_t cols) { return ((size_t)bwd_blocks(rows, cols) * (size_t)cols * 4 + 255) / 256 * 256; }

#define STX_NORM_GO(KERNEL, T, BLOCKS)                                                                              \
    do {                                                                                                            \
        const int64_t n = a.cols;                                                                                   \
        if (n <= 128) hipLaunchKernelGGL((KERNEL<T, 16, 1>), dim3(BLOCKS), dim3(kThreads), 0, c->stream, a);        \
        else if (n <= 256) hipLaunchKernelGGL((KERNEL<T, 32, 1>), dim3(BLOCKS), dim3(kThreads), 0, c->stream, a);   \
        else if (n <= 512) hipLaunchKernelGGL((KERNEL<T, 64, 1>), dim3(BLOCKS), dim3(kThreads), 0, c->stream, a);   \
        else if (n <= 1024) hipLaunchKernelGGL((KERNEL<T, 64, 2>), dim3(BLOCKS), dim3(kThreads), 0, c->stream, a);  \
        else if (n <= 2048) hipLaunchKernelGGL((KERNEL<T, 64, 4>), dim3(BLOCKS), dim3(kThreads), 0, c->stream, a);  \
        else if (n <= 4096) hipLaunchKernelGGL((KERNEL<T, 256, 2>), dim3(BLOCKS), dim3(kThreads), 0, c->stream, a); \
        else if (n <= 8192) hipLaunchKernelGGL((KERNEL<T, 256, 4>), dim3(BLOCKS), dim3(kThreads), 0, c->stream, a); \
        else hipLaunchKernelGGL((KERNEL<T, 256, 8>), dim3(BLOCKS), dim3(kThreads), 0, c->stream, a);                \
    } while (0)
#define STX_NORM_TYPE(KERNEL, BLOCKS)                                     \
    do {                                                                  \
        if (dtype == STX_F32) STX_NORM_GO(KERNEL, float, BLOCKS);         \
        else if (dtype == STX_BF16) STX_NORM_GO(KERNEL, bf16_t, BLOCKS);  \
        else STX_NORM_GO(KERNEL, f16_t, BLOCKS);                          \
    } while (0)

stx_status launch_rmsnorm(stx_ctx *c, int dtype, const NormArgs &a)
{
    const int64_t groups = kThreads / row_threads(a.cols);
    const unsigned blocks = (unsigned)((a.rows + groups - 1) / groups);
    ProfScope prof(c, "k_rmsnorm");
    STX_NORM_TYPE(k_rmsnorm, blocks);
    return hip_ok(hipGetLastError());
}

stx_status launch_rmsnorm_backward(stx_ctx *c, int dtype, const NormBwdArgs &a, float *dweight)
{
    const unsigned blocks = (unsigned)bwd_blocks(a.rows, a.cols);
    if (blocks) {
        ProfScope prof(c, "k_rmsnorm_bwd");
        STX_NORM_TYPE(k_rmsnorm_bwd, blocks);
    }
    if (dweight) {
        ProfScope prof(c, "k_norm_dweight");
        hipLaunchKernelGGL(k_norm_dweight, dim3((unsigned)((a.cols + 15) / 16)), dim3(kThreads), 0, c->stream, a.partials, (int)blocks,
                           a.cols, dweight);
    }
    return hip_ok(hipGetLastError());
}

}  // namespace stx
