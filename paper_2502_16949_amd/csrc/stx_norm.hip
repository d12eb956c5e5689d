// Root-mean-square norm of rows with the residual's addition, its 8-bit output, and its backward pass.
//
//   s = x + residual (rounded to the rows' type);  y = s rstd w,  rstd = (mean(s^2) + eps)^-1/2
//   a = dy w;  dx = rstd (a - s rstd^2 mean(a s)) + dsum;  dw = sum_rows dy s rstd
//
// Both directions are bound by memory: a row is read once, held in registers as floats while its sum is formed, and written
// once.  G threads share a row, an octet (stx_fp8.h) each, and two of them above 8,192 columns: up to 512 columns a part of a
// wavefront, whose sum needs no barrier.  (Two octets each up to 1,024 columns, to need no barrier there either, leave fewer
// wavefronts to wait for memory: 20,011 fp32 rows of 1,001 with a residual in 75 us, so in 64.)
#include "stx_device.h"
#include "stx_fp8.h"
#include "stx_internal.h"
#include "stx_ops.h"

namespace stx {

constexpr int row_block(int g) { return g < kThreads ? kThreads : g; }     // threads of a workgroup

// Sum over the G threads that share a row; every one receives it.  Above a wavefront: through s_red[slot], where calls in turn
// take slots in turn.
template <int G>
__device__ inline float row_sum(float v, float (*s_red)[16], int slot)
{
    if constexpr (G <= 64) return group_sum<G>(v);
    else {
        v = group_sum<64>(v);
        float *mine = s_red[slot] + threadIdx.x / G * (G / 64);       // (128 threads: two rows in a workgroup)
        if ((threadIdx.x & 63) == 0) mine[(threadIdx.x % G) >> 6] = v;
        __syncthreads();
        return group_sum<G / 64>(mine[threadIdx.x % (G / 64)]);
    }
}

template <class T, int G, int ITERS>
__global__ __launch_bounds__(row_block(G)) void k_rmsnorm(NormArgs a)
{
    constexpr int GROUPS = row_block(G) / G;
    __shared__ float s_red[1][16];
    const int g = threadIdx.x % G, l16 = g & 15;
    const int64_t mine = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
    if (G != 128 && mine >= a.rows) return;
    const bool in = G != 128 || mine < a.rows;               // two rows share a workgroup's barriers: one behind the end goes along
    const int64_t row = G != 128 ? mine : min(mine, a.rows - 1), at = row * a.ld;
    const T *x = (const T *)a.x + at, *res = a.residual ? (const T *)a.residual + at : nullptr;
    T *sum = in && a.sum ? (T *)a.sum + at : nullptr;
    Octet<T> xo[ITERS], ro[ITERS];
    float s[ITERS][8], ss = 0.f;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) xo[it] = request_octet(x, (it * G + g) >> 4, l16, a.cols);
    if (res) {
#pragma unroll
        for (int it = 0; it < ITERS; ++it) ro[it] = request_octet(res, (it * G + g) >> 4, l16, a.cols);
    }
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        octet_floats(xo[it], (it * G + g) >> 4, l16, a.cols, s[it]);
        if (res) {
            float r[8];
            octet_floats(ro[it], (it * G + g) >> 4, l16, a.cols, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[it][j] += r[j];
        }
    }
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        round_store_octet<T>(sum, (it * G + g) >> 4, l16, a.cols, s[it], a.past);
#pragma unroll
        for (int j = 0; j < 8; ++j) ss += s[it][j] * s[it][j];
    }
    if (!a.y && !a.q.codes && !a.rstd) return;
    const float rstd = 1.0f / sqrtf(row_sum<G>(ss, s_red, 0) / (float)a.cols + a.eps);
    if (!in) return;
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
            if (octet_pos<T>(blk, l16, 7) >= a.cols) {       // behind the row's end: 0 times an rstd or weight that need not be finite
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (octet_pos<T>(blk, l16, j) >= a.cols) s[it][j] = 0.f;
            }
            if (a.format == STX_E4M3) store_q8_octet<T, STX_E4M3>(a.q, row, blk, l16, s[it]);
            else store_q8_octet<T, STX_E5M2>(a.q, row, blk, l16, s[it]);
        }
        if (a.y) round_store_octet<T>((T *)a.y + at, blk, l16, a.cols, s[it], a.past);
    }
}

// A workgroup takes rows in turn and keeps its part of dweight in registers; the parts are joined by k_norm_dweight.
// (Four wavefronts a SIMD: every workgroup of the grid is resident.  The next row is requested before this one is reckoned:
// 32,768 bf16 rows of 1,024 in 65 us, so in 55.  Above 8,192 columns the sum's weights and dsum are read where they are used.)
template <class T, int G, int ITERS>
__global__ __launch_bounds__(row_block(G), 4) void k_rmsnorm_bwd(NormBwdArgs a)
{
    constexpr int GROUPS = row_block(G) / G;
    __shared__ float s_red[2][16];
    __shared__ float s_dw[GROUPS > 1 ? GROUPS * G * 8 : 1];
    const int g = threadIdx.x % G, grp = threadIdx.x / G, l16 = g & 15;
    float w[8], dw[ITERS][8];              // (two octets each: the weight is read again for every row, there are no registers for it)
    auto weight = [&](int it) {
        if (a.weight) load_octet_as<T>(a.weight, (it * G + g) >> 4, l16, a.cols, w);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = 1.f;
    };
    if (ITERS == 1) weight(0);
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[it][j] = 0.f;
    struct Row { Octet<T> s[ITERS], d[ITERS], e; float rstd; };
    auto request = [&](int64_t row, Row &r) {
        const int64_t at = row * a.ld;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            r.s[it] = request_octet((const T *)a.sum + at, (it * G + g) >> 4, l16, a.cols);
            r.d[it] = request_octet((const T *)a.dy + at, (it * G + g) >> 4, l16, a.cols);
        }
        if (ITERS == 1 && a.dsum) r.e = request_octet((const T *)a.dsum + at, g >> 4, l16, a.cols);
        r.rstd = a.rstd[row];
    };
    const int64_t stride = (int64_t)gridDim.x * GROUPS, last = a.rows - 1;
    int slot = 0;
    Row r;
    if (ITERS == 1) request(min((int64_t)blockIdx.x * GROUPS + grp, last), r);
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < a.rows; first += stride, slot ^= 1) {
        const int64_t row = first + grp;
        const bool in = row < a.rows;      // (rows that share a workgroup's barriers go along behind the end)
        Row next;
        if (ITERS == 1 && first + stride < a.rows) request(min(row + stride, last), next);     // under way meanwhile
        if (ITERS > 1) request(row, r);
        float s[ITERS][8], d[ITERS][8], dot = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            octet_floats(r.s[it], (it * G + g) >> 4, l16, a.cols, s[it]);
            octet_floats(r.d[it], (it * G + g) >> 4, l16, a.cols, d[it]);
            if (ITERS > 1) weight(it);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (in) dw[it][j] += d[it][j] * (s[it][j] * r.rstd);
                d[it][j] *= w[j];
                dot += d[it][j] * s[it][j];
            }
        }
        const float c = row_sum<G>(dot, s_red, slot) / (float)a.cols * r.rstd * r.rstd;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            float e[8];
            if (a.dsum) {
                if (ITERS > 1) r.e = request_octet((const T *)a.dsum + row * a.ld, (it * G + g) >> 4, l16, a.cols);
                octet_floats(r.e, (it * G + g) >> 4, l16, a.cols, e);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                d[it][j] = (d[it][j] - s[it][j] * c) * r.rstd;
                if (a.dsum) d[it][j] += e[j];
            }
            if (in) round_store_octet<T>((T *)a.dx + row * a.ld, (it * G + g) >> 4, l16, a.cols, d[it], a.past);
        }
        if (ITERS == 1) r = next;          // (two octets each leave no registers for a second row)
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

// dweight = the workgroups' parts, 64 slices of them side by side and then in order, in 64 bits: in 32 these up to 1,024 numbers
// cost more of the result than everything before them (20,011 fp32 rows of 1,001: 1.4e-7 of it in all, so 9e-8).
__global__ __launch_bounds__(1024) void k_norm_dweight(const float *__restrict__ partials, int n, int64_t cols, float *__restrict__ dweight)
{
    __shared__ double s_part[64][17];
    const int c = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int64_t col = (int64_t)blockIdx.x * 16 + c;
    double t = 0.0;
    if (col < cols) {
#pragma unroll 4
        for (int i = slice; i < n; i += 64) t += partials[(int64_t)i * cols + col];
    }
    s_part[slice][c] = t;
    __syncthreads();
    if (slice < 8) {
#pragma unroll
        for (int u = 1; u < 8; ++u) t += s_part[slice + 8 * u][c];
        s_part[slice][c] = t;
    }
    __syncthreads();
    if (slice == 0 && col < cols) {
#pragma unroll
        for (int u = 1; u < 8; ++u) t += s_part[u][c];
        dweight[col] = (float)t;
    }
}

static int row_threads(int64_t cols)
{
    int g = 16;
    while (g < 1024 && g * 8 < cols) g *= 2;
    return g;
}

// Workgroups of a backward pass: as many as are resident, so that each sums many rows into its part.
static int bwd_blocks(int64_t rows, int64_t cols)
{
    const int g = row_threads(cols);
    const int64_t groups = row_block(g) / g, need = (rows + groups - 1) / groups, most = 256 * 1024 / row_block(g);
    return (int)(need < most ? need : most);
}
size_t norm_bwd_work_bytes(int64_t rows, int64_t cols) { return ((size_t)bwd_blocks(rows, cols) * (size_t)cols * 4 + 255) / 256 * 256; }

#define STX_NORM_GO(KERNEL, T, BLOCKS)                                                                            \
    do {                                                                                                          \
        const int64_t n = a.cols;                                                                                 \
        if (n <= 128) hipLaunchKernelGGL((KERNEL<T, 16, 1>), dim3(BLOCKS), dim3(256), 0, c->stream, a);           \
        else if (n <= 256) hipLaunchKernelGGL((KERNEL<T, 32, 1>), dim3(BLOCKS), dim3(256), 0, c->stream, a);      \
        else if (n <= 512) hipLaunchKernelGGL((KERNEL<T, 64, 1>), dim3(BLOCKS), dim3(256), 0, c->stream, a);      \
        else if (n <= 1024) hipLaunchKernelGGL((KERNEL<T, 128, 1>), dim3(BLOCKS), dim3(256), 0, c->stream, a);    \
        else if (n <= 2048) hipLaunchKernelGGL((KERNEL<T, 256, 1>), dim3(BLOCKS), dim3(256), 0, c->stream, a);    \
        else if (n <= 4096) hipLaunchKernelGGL((KERNEL<T, 512, 1>), dim3(BLOCKS), dim3(512), 0, c->stream, a);    \
        else if (n <= 8192) hipLaunchKernelGGL((KERNEL<T, 1024, 1>), dim3(BLOCKS), dim3(1024), 0, c->stream, a);  \
        else hipLaunchKernelGGL((KERNEL<T, 1024, 2>), dim3(BLOCKS), dim3(1024), 0, c->stream, a);                 \
    } while (0)
#define STX_NORM_TYPE(KERNEL, BLOCKS)                                    \
    do {                                                                 \
        if (dtype == STX_F32) STX_NORM_GO(KERNEL, float, BLOCKS);        \
        else if (dtype == STX_BF16) STX_NORM_GO(KERNEL, bf16_t, BLOCKS); \
        else STX_NORM_GO(KERNEL, f16_t, BLOCKS);                         \
    } while (0)

// Rows of whole lines beyond the caches go past them: 20,011 x 1,024 fp32 with a residual 55.4 us in place of 59.7, backward 65.3 and
// 67.9; 32,768 x 1,024 bf16 into 8 bits 43.2 and 45.1.  (Rows that leave parts of lines: 20,011 x 1,001 fp32 66.5 us, and 62.8 so.)
static bool past_caches(const void *out, int64_t rows, int64_t ld, int64_t size)
{
    return rows * ld * size >= ((int64_t)64 << 20) && ld * size % 128 == 0 && (uintptr_t)out % 128 == 0;
}

stx_status launch_rmsnorm(stx_ctx *c, int dtype, const NormArgs &all)
{
    const int g = row_threads(all.cols);
    const int64_t groups = row_block(g) / g, most = kMaxItems / row_block(g) * groups, e = dtype == STX_F32 ? 4 : 2;
    NormArgs a = all;
    a.past = past_caches(a.sum ? a.sum : a.y, a.rows, a.ld, e);
    auto behind = [&](void *p) { return p ? (char *)p + most * a.ld * e : nullptr; };
    for (int64_t left = all.rows; left > 0; left -= most) {  // (one launch but for 16 million wide rows)
        a.rows = left < most ? left : most;
        const unsigned blocks = (unsigned)((a.rows + groups - 1) / groups);
        {
            ProfScope prof(c, "k_rmsnorm");
            STX_NORM_TYPE(k_rmsnorm, blocks);
        }
        if (left <= most) break;
        a.x = behind((void *)a.x);
        a.residual = behind((void *)a.residual);
        a.sum = behind(a.sum);
        a.y = behind(a.y);
        if (a.rstd) a.rstd += most;
        if (a.q.codes) {
            a.q.codes += most * a.q.ld;
            a.q.scales += most * a.q.ld_scale;
        }
    }
    return hip_ok(hipGetLastError());
}

stx_status launch_rmsnorm_backward(stx_ctx *c, int dtype, const NormBwdArgs &all, float *dweight)
{
    NormBwdArgs a = all;
    a.past = past_caches(a.dx, a.rows, a.ld, dtype == STX_F32 ? 4 : 2);
    const unsigned blocks = (unsigned)bwd_blocks(a.rows, a.cols);
    if (blocks) {
        ProfScope prof(c, "k_rmsnorm_bwd");
        STX_NORM_TYPE(k_rmsnorm_bwd, blocks);
    }
    if (dweight) {
        ProfScope prof(c, "k_norm_dweight");
        hipLaunchKernelGGL(k_norm_dweight, dim3((unsigned)((a.cols + 15) / 16)), dim3(1024), 0, c->stream, a.partials, (int)blocks,
                           a.cols, dweight);
    }
    return hip_ok(hipGetLastError());
}

}  // namespace stx
