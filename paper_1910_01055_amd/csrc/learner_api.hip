// Entry points of the learner's operators: checks of the arguments, then the launchers.
#include "learner.hpp"

using namespace aq;

namespace {

constexpr int64_t kMostRows = 0x7fffffffLL, kMostCols = 1LL << 20, kMostLd = 1LL << 21;

hipStream_t as_stream(void* s) { return (hipStream_t)s; }

// AQ_OK, or what is wrong with one operand
aq_status matrix_ok(const aq_matrix* m) {
    if (!m || m->rows < 0 || m->cols < 0 || m->ld < m->cols) return AQ_EINVAL;
    if (m->dtype != AQ_F32 && m->dtype != AQ_F16 && m->dtype != AQ_BF16) return AQ_EINVAL;
    if (!m->d && m->rows > 0) return AQ_EINVAL;
    if ((uintptr_t)m->d % dtype_bytes(m->dtype)) return AQ_EINVAL;
    if (m->rows > kMostRows || m->cols < 1 || m->cols > kMostCols || m->ld > kMostLd) return AQ_ESHAPE;
    return AQ_OK;
}
template <class Blocks32>
aq_status blocks_ok(const Blocks32* b) {
    if (!b || b->rows < 0 || b->cols < 0) return AQ_EINVAL;
    if ((!b->d_codes || !b->d_scales) && b->rows > 0) return AQ_EINVAL;
    if ((uintptr_t)b->d_codes & 15) return AQ_EINVAL;
    if (b->rows > kMostRows || b->cols < 1 || b->cols > kMostCols) return AQ_ESHAPE;
    return AQ_OK;
}
bool floats_ok(const void* p) { return ((uintptr_t)p & 3) == 0; }
aq_status sizes_ok(int64_t rows, int64_t n, int64_t k, const uint64_t* bytes) {
    if (!bytes || rows < 0 || n < 0 || k < 0) return AQ_EINVAL;
    return rows > kMostRows || n < 1 || n > kMostCols || k < 1 || k > kMostCols ? AQ_ESHAPE : AQ_OK;
}

}  // namespace

#define AQ_TRY(expr)                       \
    do {                                   \
        const aq_status tried = (expr);    \
        if (tried != AQ_OK) return tried;  \
    } while (0)

extern "C" aq_status aq_layernorm_forward(const aq_matrix* x, const float* d_gamma, const float* d_beta, float eps, const aq_matrix* y,
                                          float* d_mean, float* d_rstd, const aq_ckpt8* kept, void* stream) {
    AQ_TRY(matrix_ok(x));
    AQ_TRY(matrix_ok(y));
    if (kept) AQ_TRY(blocks_ok(kept));
    if (!floats_ok(d_gamma) || !floats_ok(d_beta) || !floats_ok(d_mean) || !floats_ok(d_rstd) || !(eps >= 0.0f)) return AQ_EINVAL;
    if (x->cols > AQ_LAYERNORM_MAX_COLS || y->rows != x->rows || y->cols != x->cols || y->dtype != x->dtype) return AQ_ESHAPE;
    if (kept && (kept->rows != x->rows || kept->cols != x->cols)) return AQ_ESHAPE;
    if (x->rows == 0) return AQ_OK;
    return launch_layernorm_forward(*x, d_gamma, d_beta, eps, *y, d_mean, d_rstd, kept, as_stream(stream));
}

extern "C" aq_status aq_layernorm_backward_workspace(int64_t rows, int64_t cols, uint64_t* bytes) {
    AQ_TRY(sizes_ok(rows, 1, cols, bytes));
    if (cols > AQ_LAYERNORM_MAX_COLS) return AQ_ESHAPE;
    *bytes = (uint64_t)layernorm_backward_workspace(rows, cols);
    return AQ_OK;
}

extern "C" aq_status aq_layernorm_backward(const aq_matrix* dy, const aq_matrix* x, const aq_ckpt8* kept, const float* d_gamma,
                                           const float* d_mean, const float* d_rstd, const aq_matrix* dx, float* d_dgamma,
                                           float* d_dbeta, void* d_workspace, uint64_t workspace_bytes, void* stream) {
    AQ_TRY(matrix_ok(dy));
    AQ_TRY(matrix_ok(dx));
    if ((x != nullptr) == (kept != nullptr)) return AQ_EINVAL;
    if (x) AQ_TRY(matrix_ok(x));
    if (kept) AQ_TRY(blocks_ok(kept));
    if (dy->rows > 0 && (!d_mean || !d_rstd)) return AQ_EINVAL;
    if (!floats_ok(d_gamma) || !floats_ok(d_mean) || !floats_ok(d_rstd) || !floats_ok(d_dgamma) || !floats_ok(d_dbeta)) return AQ_EINVAL;
    if (dy->cols > AQ_LAYERNORM_MAX_COLS || dx->rows != dy->rows || dx->cols != dy->cols || dx->dtype != dy->dtype) return AQ_ESHAPE;
    if (x && (x->rows != dy->rows || x->cols != dy->cols || x->dtype != dy->dtype)) return AQ_ESHAPE;
    if (kept && (kept->rows != dy->rows || kept->cols != dy->cols)) return AQ_ESHAPE;
    if (!workspace_ok(d_workspace, workspace_bytes, layernorm_backward_workspace(dy->rows, dy->cols))) return AQ_EINVAL;
    return launch_layernorm_backward(*dy, x, kept, d_gamma, d_mean, d_rstd, *dx, d_dgamma, d_dbeta, (float*)d_workspace, as_stream(stream));
}

extern "C" aq_status aq_ckpt8_pack(const aq_matrix* x, const aq_ckpt8* kept, void* stream) {
    AQ_TRY(matrix_ok(x));
    AQ_TRY(blocks_ok(kept));
    if (kept->rows != x->rows || kept->cols != x->cols) return AQ_ESHAPE;
    return x->rows == 0 ? AQ_OK : launch_ckpt8_pack(*x, *kept, as_stream(stream));
}

extern "C" aq_status aq_ckpt8_unpack(const aq_ckpt8* kept, const aq_matrix* x, void* stream) {
    AQ_TRY(blocks_ok(kept));
    AQ_TRY(matrix_ok(x));
    if (kept->rows != x->rows || kept->cols != x->cols) return AQ_ESHAPE;
    return x->rows == 0 ? AQ_OK : launch_ckpt8_unpack(*kept, *x, as_stream(stream));
}

extern "C" aq_status aq_ckpt8_weight_grad_workspace(int64_t rows, int64_t n, int64_t k, uint64_t* bytes) {
    AQ_TRY(sizes_ok(rows, n, k, bytes));
    *bytes = (uint64_t)weight_grad_workspace(rows, n, k);
    return AQ_OK;
}

extern "C" aq_status aq_ckpt8_weight_grad(const aq_matrix* dy, const aq_ckpt8* kept, const aq_matrix* dw, float* d_db, void* d_workspace,
                                          uint64_t workspace_bytes, void* stream) {
    AQ_TRY(matrix_ok(dy));
    AQ_TRY(blocks_ok(kept));
    AQ_TRY(matrix_ok(dw));
    if (!floats_ok(d_db)) return AQ_EINVAL;
    if (kept->rows != dy->rows || dw->rows != dy->cols || dw->cols != kept->cols || dw->dtype != AQ_F32) return AQ_ESHAPE;
    return launch_weight_grad(*dy, *kept, *dw, d_db, d_workspace, workspace_bytes, as_stream(stream));
}

extern "C" aq_status aq_mx4_quantize(const aq_matrix* x, const aq_mx4* q, void* stream) {
    AQ_TRY(matrix_ok(x));
    AQ_TRY(blocks_ok(q));
    if (q->rows != x->rows || q->cols != x->cols) return AQ_ESHAPE;
    return x->rows == 0 ? AQ_OK : launch_mx4_quantize(*x, *q, as_stream(stream));
}

extern "C" aq_status aq_mx4_dequantize(const aq_mx4* q, const aq_matrix* x, void* stream) {
    AQ_TRY(blocks_ok(q));
    AQ_TRY(matrix_ok(x));
    if (q->rows != x->rows || q->cols != x->cols) return AQ_ESHAPE;
    return x->rows == 0 ? AQ_OK : launch_mx4_dequantize(*q, *x, as_stream(stream));
}

extern "C" aq_status aq_mx4_linear_workspace(int64_t rows, int64_t n, int64_t k, uint64_t* bytes) {
    AQ_TRY(sizes_ok(rows, n, k, bytes));
    *bytes = (uint64_t)mx4_linear_workspace(rows, n, k);
    return AQ_OK;
}

extern "C" aq_status aq_mx4_linear(const aq_matrix* x, const aq_mx4* w, const float* d_bias, const aq_matrix* y, void* d_workspace,
                                   uint64_t workspace_bytes, void* stream) {
    AQ_TRY(matrix_ok(x));
    AQ_TRY(blocks_ok(w));
    AQ_TRY(matrix_ok(y));
    if (!floats_ok(d_bias)) return AQ_EINVAL;
    if (w->cols != x->cols || y->rows != x->rows || y->cols != w->rows || y->dtype != x->dtype) return AQ_ESHAPE;
    if (!workspace_ok(d_workspace, workspace_bytes, mx4_linear_workspace(x->rows, w->rows, w->cols))) return AQ_EINVAL;
    return x->rows == 0 ? AQ_OK : launch_mx4_linear(*x, *w, d_bias, *y, d_workspace, as_stream(stream));
}

extern "C" aq_status aq_mx4_matmul(const aq_mx4* x, const aq_mx4* w, const float* d_bias, const aq_matrix* y, void* stream) {
    AQ_TRY(blocks_ok(x));
    AQ_TRY(blocks_ok(w));
    AQ_TRY(matrix_ok(y));
    if (!floats_ok(d_bias)) return AQ_EINVAL;
    if (w->cols != x->cols || y->rows != x->rows || y->cols != w->rows) return AQ_ESHAPE;
    return x->rows == 0 ? AQ_OK : launch_mx4_matmul(*x, *w, d_bias, *y, as_stream(stream));
}

extern "C" aq_status aq_mx4_input_grad_workspace(int64_t rows, int64_t n, int64_t k, uint64_t* bytes) {
    AQ_TRY(sizes_ok(rows, n, k, bytes));
    *bytes = (uint64_t)input_grad_workspace(rows, n, k);
    return AQ_OK;
}

extern "C" aq_status aq_mx4_input_grad(const aq_matrix* dy, const aq_mx4* w, const aq_matrix* dx, void* d_workspace, uint64_t workspace_bytes,
                                       void* stream) {
    AQ_TRY(matrix_ok(dy));
    AQ_TRY(blocks_ok(w));
    AQ_TRY(matrix_ok(dx));
    if (w->rows != dy->cols || dx->rows != dy->rows || dx->cols != w->cols || dx->dtype != dy->dtype) return AQ_ESHAPE;
    return dy->rows == 0 ? AQ_OK : launch_input_grad(*dy, *w, *dx, d_workspace, workspace_bytes, as_stream(stream));
}
