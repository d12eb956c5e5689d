// Launchers of the operators that work on plain rows and tensors (8-bit rows and products, RMS norm, AdamW): what the C entry
// points of stx_ops.cpp hand to stx_norm.hip, stx_q8.hip, stx_q8_matmul.hip and stx_adamw.hip.
#pragma once

#include "stx_fp8.h"
#include "stx_internal.h"

namespace stx {

constexpr int64_t kNormMaxCols = 16384;
constexpr int64_t kMaxItems = ((int64_t)1 << 32) - 1;      // work items of one launch

struct NormArgs {
    const void *x, *residual;
    const float *weight;
    float eps;
    void *sum, *y;
    Q8Out q;
    int32_t format;
    float *rstd;
    int64_t rows, cols, ld;
    bool past;                             // (set by the launcher)
};
struct NormBwdArgs {
    const void *sum;
    const float *weight, *rstd;
    const void *dy, *dsum;
    void *dx;
    float *partials;                       // [workgroups][cols], or null
    int64_t rows, cols, ld;
    bool past;                             // (set by the launcher)
};
stx_status launch_rmsnorm(stx_ctx *, int dtype, const NormArgs &);
size_t norm_bwd_work_bytes(int64_t rows, int64_t cols);
stx_status launch_rmsnorm_backward(stx_ctx *, int dtype, const NormBwdArgs &, float *dweight);

stx_status launch_q8_quantize(stx_ctx *, int dtype, int64_t rows, int64_t cols, int64_t ld, const void *x, const stx_q8 *q,
                              const stx_q8 *qt);

size_t q8_matmul_work_bytes(int64_t m, int64_t n, int64_t k);
stx_status launch_q8_matmul(stx_ctx *, const stx_q8 *a, const stx_q8 *b, int dtype, void *out, int64_t ldo, void *work);

stx_status launch_adamw_tensors(stx_ctx *, const stx_adamw *, const stx_adamw_tensor *, int n);
stx_status launch_adamw_step(stx_ctx *, stx_params *, const stx_incidence *, const stx_grads *, const stx_adamw *,
                             const stx_adamw_state *);

}  // namespace stx
