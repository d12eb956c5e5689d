// C entry points of the operators on plain rows and tensors: argument checks and dispatch (stx_api.cpp holds those of the
// training step).
#include "stx_ops.h"

using namespace stx;

namespace {

constexpr int64_t kMaxIndex = ((int64_t)1 << 31) - 1;

bool row_dtype(int32_t d) { return d == STX_F32 || d == STX_BF16 || d == STX_F16; }
uintptr_t element(int32_t d) { return d == STX_F32 ? 4u : 2u; }
bool aligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// A matrix in 8 bits of the given size (null is the caller's business).
stx_status check_q8(const stx_q8 *q, int64_t rows, int64_t cols)
{
    if (q->rows != rows || q->cols != cols || rows < 0 || cols < 0 || rows > kMaxIndex || cols > kMaxIndex - kBlock) return STX_ERR_BAD_ARG;
    if (q->format != STX_E4M3 && q->format != STX_E5M2) return STX_ERR_BAD_ARG;
    if (rows == 0 || cols == 0) return STX_OK;
    if (!q->codes || !q->scales) return STX_ERR_NULL;
    const int64_t blocks = (cols + kBlock - 1) / kBlock;
    if (q->ld % 16 != 0 || q->ld < blocks * kBlock || q->ld_scale % 4 != 0 || q->ld_scale < blocks) return STX_ERR_BAD_ARG;
    if (!aligned(q->codes, 16) || !aligned(q->scales, 4)) return STX_ERR_BAD_ARG;
    return STX_OK;
}

stx_status check_adamw(const stx_adamw *h)
{
    if (!h) return STX_ERR_NULL;
    if (h->bits != 32 && h->bits != 8) return STX_ERR_BAD_ARG;
    if (!(h->lr == h->lr) || !(h->weight_decay == h->weight_decay)) return STX_ERR_BAD_ARG;
    if (!(h->beta1 >= 0.0 && h->beta1 < 1.0) || !(h->beta2 >= 0.0 && h->beta2 < 1.0) ||
        !(h->eps == 0.0 || (h->eps >= 0x1p-126 && h->eps <= 0x1p126))) return STX_ERR_BAD_ARG;
    if (!h->step_dev && h->step < 1) return STX_ERR_BAD_ARG;
    if (!aligned(h->step_dev, 8) || !aligned(h->grad_scale, 4)) return STX_ERR_BAD_ARG;
    return STX_OK;
}

stx_status check_moments(const stx_moments &s, int bits, uintptr_t align)
{
    if (!s.m || !s.v) return STX_ERR_NULL;
    if (bits == 8 && (!s.m_scale || !s.v_scale)) return STX_ERR_NULL;
    const uintptr_t a = bits == 8 ? (align + 3) / 4 : align;
    if (!aligned(s.m, a) || !aligned(s.v, a)) return STX_ERR_BAD_ARG;
    if (bits == 8 && (!aligned(s.m_scale, 4) || !aligned(s.v_scale, 4))) return STX_ERR_BAD_ARG;
    return STX_OK;
}

}  // namespace

extern "C" {

stx_status stx_rmsnorm(stx_ctx *ctx, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const void *x, const void *residual,
                       const float *weight, float eps, void *sum, void *y, const stx_q8 *q, float *rstd)
{
    if (!ctx) return STX_ERR_NULL;
    if (!row_dtype(dtype) || rows < 0 || rows > kMaxIndex || cols < 1 || cols > kNormMaxCols || ld < cols) return STX_ERR_BAD_ARG;
    if (!(eps >= 0.0f)) return STX_ERR_BAD_ARG;
    if (q) {
        const stx_status s = check_q8(q, rows, cols);
        if (s != STX_OK) return s;
    }
    if (rows == 0) return STX_OK;
    if (!x || (!sum && !y && !q && !rstd)) return STX_ERR_NULL;
    const uintptr_t e = element(dtype);
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(sum, e) || !aligned(y, e) || !aligned(weight, 4) || !aligned(rstd, 4))
        return STX_ERR_BAD_ARG;
    const NormArgs a{x, residual, weight, eps, sum, y, q ? Q8Out{q->codes, q->scales, q->ld, q->ld_scale} : Q8Out{}, q ? q->format : 0,
                     rstd, rows, cols, ld, false};
    return launch_rmsnorm(ctx, dtype, a);
}

stx_status stx_rmsnorm_backward_work_bytes(const stx_ctx *ctx, int64_t rows, int64_t cols, size_t *bytes)
{
    if (!ctx || !bytes) return STX_ERR_NULL;
    if (rows < 0 || rows > kMaxIndex || cols < 1 || cols > kNormMaxCols) return STX_ERR_BAD_ARG;
    *bytes = norm_bwd_work_bytes(rows, cols);
    return STX_OK;
}

stx_status stx_rmsnorm_backward(stx_ctx *ctx, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const void *sum,
                                const float *weight, const float *rstd, const void *dy, const void *dsum, void *dx, float *dweight,
                                void *work, size_t work_bytes)
{
    if (!ctx) return STX_ERR_NULL;
    if (!row_dtype(dtype) || rows < 0 || rows > kMaxIndex || cols < 1 || cols > kNormMaxCols || ld < cols) return STX_ERR_BAD_ARG;
    const uintptr_t e = element(dtype);
    if (!aligned(sum, e) || !aligned(dy, e) || !aligned(dsum, e) || !aligned(dx, e) || !aligned(weight, 4) || !aligned(rstd, 4) ||
        !aligned(dweight, 4))
        return STX_ERR_BAD_ARG;
    if (rows > 0 && (!sum || !rstd || !dy || !dx)) return STX_ERR_NULL;
    const size_t need = dweight ? norm_bwd_work_bytes(rows, cols) : 0;
    if (need > 0 && !work) return STX_ERR_NULL;
    if (need > 0 && (work_bytes < need || !aligned(work, 256))) return STX_ERR_WORKSPACE;
    if (rows == 0 && !dweight) return STX_OK;
    const NormBwdArgs a{sum, weight, rstd, dy, dsum, dx, dweight ? (float *)work : nullptr, rows, cols, ld, false};
    return launch_rmsnorm_backward(ctx, dtype, a, dweight);
}

stx_status stx_q8_quantize(stx_ctx *ctx, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const void *x, const stx_q8 *q,
                           const stx_q8 *qt)
{
    if (!ctx) return STX_ERR_NULL;
    if (!row_dtype(dtype) || rows < 0 || rows > kMaxIndex || cols < 0 || cols > kMaxIndex || ld < cols) return STX_ERR_BAD_ARG;
    if (!q && !qt) return STX_ERR_NULL;
    stx_status s = q ? check_q8(q, rows, cols) : STX_OK;
    if (s == STX_OK && qt) s = check_q8(qt, cols, rows);
    if (s != STX_OK) return s;
    if (rows == 0 || cols == 0) return STX_OK;
    if (!x) return STX_ERR_NULL;
    if (!aligned(x, element(dtype))) return STX_ERR_BAD_ARG;
    const int64_t cb = (cols + kBlock - 1) / kBlock, rb = (rows + kBlock - 1) / kBlock;
    if (rows > ((int64_t)1 << 35) / cb || (qt && rb > kMaxItems / kThreads / cb)) return STX_ERR_UNSUPPORTED;
    return launch_q8_quantize(ctx, dtype, rows, cols, ld, x, q, qt);
}

stx_status stx_q8_matmul_work_bytes(const stx_ctx *ctx, int64_t rows_a, int64_t rows_b, int64_t cols, size_t *bytes)
{
    if (!ctx || !bytes) return STX_ERR_NULL;
    if (rows_a < 0 || rows_b < 0 || cols < 1 || rows_a > kMaxIndex || rows_b > kMaxIndex || cols > kMaxIndex - kBlock) return STX_ERR_BAD_ARG;
    *bytes = q8_matmul_work_bytes(rows_a, rows_b, cols);
    return STX_OK;
}

stx_status stx_q8_matmul(stx_ctx *ctx, const stx_q8 *a, const stx_q8 *b, int32_t dtype, void *out, int64_t ldo, void *work, size_t work_bytes)
{
    if (!ctx || !a || !b) return STX_ERR_NULL;
    stx_status s = check_q8(a, a->rows, a->cols);
    if (s == STX_OK) s = check_q8(b, b->rows, b->cols);
    if (s != STX_OK) return s;
    if (a->cols != b->cols || a->cols < 1 || !row_dtype(dtype) || ldo < b->rows) return STX_ERR_BAD_ARG;
    if (a->rows == 0 || b->rows == 0) return STX_OK;
    for (const stx_q8 *q : {a, b})         // a tile's rows: 32-bit offsets
        if (q->ld > ((int64_t)1 << 24) || q->ld_scale > ((int64_t)1 << 24)) return STX_ERR_UNSUPPORTED;
    if (a->rows > ((int64_t)1 << 44) / b->rows || a->rows > ((int64_t)1 << 30) || b->rows > ((int64_t)1 << 30)) return STX_ERR_UNSUPPORTED;   // tiles of one launch
    if (!out) return STX_ERR_NULL;
    if (!aligned(out, element(dtype))) return STX_ERR_BAD_ARG;
    const size_t need = q8_matmul_work_bytes(a->rows, b->rows, a->cols);
    if (need > 0 && !work) return STX_ERR_NULL;
    if (need > 0 && (work_bytes < need || !aligned(work, 256))) return STX_ERR_WORKSPACE;
    return launch_q8_matmul(ctx, a, b, dtype, out, ldo, work);
}

stx_status stx_adamw_tensors(stx_ctx *ctx, const stx_adamw *h, const stx_adamw_tensor *tensors, int32_t n_tensors)
{
    if (!ctx) return STX_ERR_NULL;
    stx_status s = check_adamw(h);
    if (s != STX_OK) return s;
    if (n_tensors < 0 || n_tensors > 65535) return STX_ERR_BAD_ARG;
    if (n_tensors > 0 && !tensors) return STX_ERR_NULL;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const stx_adamw_tensor &t = tensors[i];
        if (t.n < 0 || t.n > ((int64_t)1 << 36) - 4096 || !row_dtype(t.g_dtype) || (t.flags & ~STX_ADAMW_NO_DECAY)) return STX_ERR_BAD_ARG;
        if (t.n == 0) continue;
        if (!t.p || !t.g) return STX_ERR_NULL;
        if (!aligned(t.p, 4) || !aligned(t.g, element(t.g_dtype))) return STX_ERR_BAD_ARG;
        if ((s = check_moments(t.s, h->bits, 4)) != STX_OK) return s;
    }
    return launch_adamw_tensors(ctx, h, tensors, n_tensors);
}

stx_status stx_adamw_step(stx_ctx *ctx, stx_params *p, const stx_incidence *inc, const stx_grads *g, const stx_adamw *h,
                          const stx_adamw_state *st)
{
    if (!ctx) return STX_ERR_NULL;
    stx_status s = check_update(ctx, p, inc, g);
    if (s != STX_OK) return s;
    if ((s = check_adamw(h)) != STX_OK) return s;
    if (!st) return STX_ERR_NULL;
    const int model = ctx->cfg.model;
    if ((s = check_moments(st->ent, h->bits, 16)) != STX_OK) return s;
    if ((model == STX_TRANSH || model == STX_TRANSR) && (s = check_moments(st->rel, h->bits, 16)) != STX_OK) return s;
    if (model == STX_TRANSH && (s = check_moments(st->w, h->bits, 16)) != STX_OK) return s;
    if (model == STX_TRANSR && (s = check_moments(st->proj, h->bits, 16)) != STX_OK) return s;
    ctx->fwd_inc = nullptr;   // the tables change: a stored forward no longer matches them
    return launch_adamw_step(ctx, p, inc, g, h, st);
}

}  // extern "C"
