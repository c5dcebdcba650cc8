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

// ---- gated layers

namespace {

// a matrix of a call whose matrices have one type
aq_status sized(const aq_matrix* m, int64_t rows, int64_t cols, int32_t dtype) {
    AQ_TRY(matrix_ok(m));
    return m->rows != rows || m->cols != cols || m->dtype != dtype ? AQ_ESHAPE : AQ_OK;
}
bool gate_ok(int32_t act) { return act >= AQ_GATE_SIGMOID && act <= AQ_GATE_RELU; }
bool dtype_ok(int32_t dtype) { return dtype == AQ_F32 || dtype == AQ_F16 || dtype == AQ_BF16; }
// rows, features and inputs whose products' tiles and laid-out pieces a launch's 32 bits count
aq_status gated_sizes_ok(int64_t rows, int64_t n, int64_t k) {
    if (rows > AQ_GATED_MAX_VALUES / (n > k ? n : k) || n > AQ_GATED_MAX_VALUES / k) return AQ_ESHAPE;
    return AQ_OK;
}

}  // namespace

extern "C" aq_status aq_gated_forward_workspace(int64_t rows, int64_t n, int64_t k, int32_t dtype, uint64_t* bytes) {
    AQ_TRY(sizes_ok(rows, n, k, bytes));
    if (!dtype_ok(dtype)) return AQ_EINVAL;
    AQ_TRY(gated_sizes_ok(rows, n, k));
    *bytes = (uint64_t)gated_forward_workspace(rows, n, k, dtype);
    return AQ_OK;
}

extern "C" aq_status aq_gated_backward_workspace(int64_t rows, int64_t n, int64_t k, int32_t dtype, uint64_t* bytes) {
    AQ_TRY(sizes_ok(rows, n, k, bytes));
    if (!dtype_ok(dtype)) return AQ_EINVAL;
    AQ_TRY(gated_sizes_ok(rows, n, k));
    *bytes = (uint64_t)gated_backward_workspace(rows, n, k, dtype);
    return AQ_OK;
}

extern "C" aq_status aq_gated_forward(const aq_matrix* x, const aq_matrix* wg, const aq_matrix* wu, int32_t act, const aq_matrix* y,
                                      const aq_matrix* gate, const aq_matrix* up, void* d_workspace, uint64_t workspace_bytes, void* stream) {
    AQ_TRY(matrix_ok(x));
    AQ_TRY(matrix_ok(wg));
    if (!gate_ok(act) || (gate != nullptr) != (up != nullptr)) return AQ_EINVAL;
    const int64_t rows = x->rows, n = wg->rows, k = x->cols;
    if (n < 1 || n > kMostCols) return AQ_ESHAPE;
    AQ_TRY(sized(wg, n, k, x->dtype));
    AQ_TRY(sized(wu, n, k, x->dtype));
    AQ_TRY(sized(y, rows, n, x->dtype));
    if (gate) {
        AQ_TRY(sized(gate, rows, n, x->dtype));
        AQ_TRY(sized(up, rows, n, x->dtype));
    }
    AQ_TRY(gated_sizes_ok(rows, n, k));
    if (!workspace_ok(d_workspace, workspace_bytes, gated_forward_workspace(rows, n, k, x->dtype))) return AQ_EINVAL;
    return rows == 0 ? AQ_OK : launch_gated_forward(*x, *wg, *wu, act, *y, gate, up, d_workspace, as_stream(stream));
}

extern "C" aq_status aq_gated_backward(const aq_matrix* dy, const aq_matrix* x, const aq_matrix* wg, const aq_matrix* wu, const aq_matrix* gate,
                                       const aq_matrix* up, int32_t act, const aq_matrix* dx, const aq_matrix* dwg, const aq_matrix* dwu,
                                       void* d_workspace, uint64_t workspace_bytes, void* stream) {
    AQ_TRY(matrix_ok(dy));
    AQ_TRY(matrix_ok(x));
    if (!gate_ok(act) || (dwg != nullptr) != (dwu != nullptr)) return AQ_EINVAL;
    const int64_t rows = x->rows, n = dy->cols, k = x->cols;
    AQ_TRY(sized(dy, rows, n, x->dtype));
    AQ_TRY(sized(wg, n, k, x->dtype));
    AQ_TRY(sized(wu, n, k, x->dtype));
    AQ_TRY(sized(gate, rows, n, x->dtype));
    AQ_TRY(sized(up, rows, n, x->dtype));
    if (dx) AQ_TRY(sized(dx, rows, k, x->dtype));
    if (dwg) {
        AQ_TRY(sized(dwg, n, k, x->dtype));
        AQ_TRY(sized(dwu, n, k, x->dtype));
    }
    AQ_TRY(gated_sizes_ok(rows, n, k));
    if (!workspace_ok(d_workspace, workspace_bytes, gated_backward_workspace(rows, n, k, x->dtype))) return AQ_EINVAL;
    return launch_gated_backward(*dy, *x, *wg, *wu, *gate, *up, act, dx, dwg, dwu, d_workspace, as_stream(stream));
}

// ---- the recurrence

namespace {

// the matrices of a pass: z's sizes and type
aq_status like(const aq_matrix* m, const aq_matrix* z) {
    AQ_TRY(matrix_ok(m));
    return m->rows != z->rows || m->cols != z->cols || m->dtype != z->dtype ? AQ_ESHAPE : AQ_OK;
}
// offsets of sequences, or equal parts of all rows
aq_status sequences_ok(const aq_matrix* z, const int32_t* offsets, int64_t count) {
    if (count < 0 || ((uintptr_t)offsets & 3)) return AQ_EINVAL;
    // (32 bits count a launch's threads, up to eight to a unit)
    if (count > kMostRows || count * z->cols > AQ_RECURRENCE_MAX_STATES) return AQ_ESHAPE;
    return !offsets && count > 0 && z->rows % count ? AQ_ESHAPE : AQ_OK;
}

}  // namespace

extern "C" aq_status aq_recurrence_workspace(int64_t rows, int64_t count, int64_t cols, uint64_t* bytes) {
    AQ_TRY(sizes_ok(rows, 1, cols, bytes));
    if (count < 0) return AQ_EINVAL;
    if (count > kMostRows || count * cols > AQ_RECURRENCE_MAX_STATES) return AQ_ESHAPE;
    *bytes = (uint64_t)recurrence_workspace(rows, count, cols);
    return AQ_OK;
}

extern "C" aq_status aq_recurrence_forward(const aq_matrix* z, const aq_matrix* v, const int32_t* d_offsets, int64_t count,
                                           const uint8_t* d_starts, const float* d_first, const aq_matrix* y, float* d_last, void* d_workspace,
                                           uint64_t workspace_bytes, void* stream) {
    AQ_TRY(matrix_ok(z));
    AQ_TRY(like(v, z));
    AQ_TRY(like(y, z));
    AQ_TRY(sequences_ok(z, d_offsets, count));
    if (!floats_ok(d_first) || !floats_ok(d_last) || (d_first && d_first == d_last)) return AQ_EINVAL;
    if (!workspace_ok(d_workspace, workspace_bytes, recurrence_workspace(z->rows, count, z->cols))) return AQ_EINVAL;
    if (count == 0) return AQ_OK;
    return launch_recurrence_forward(*z, *v, d_offsets, count, d_starts, d_first, *y, d_last, (float*)d_workspace, as_stream(stream));
}

extern "C" aq_status aq_recurrence_backward(const aq_matrix* dy, const float* d_dlast, const aq_matrix* z, const aq_matrix* v,
                                            const aq_matrix* y, const int32_t* d_offsets, int64_t count, const uint8_t* d_starts,
                                            const float* d_first, const aq_matrix* dz, const aq_matrix* dv, float* d_dfirst, void* d_workspace,
                                            uint64_t workspace_bytes, void* stream) {
    AQ_TRY(matrix_ok(z));
    AQ_TRY(like(dy, z));
    AQ_TRY(like(v, z));
    AQ_TRY(like(y, z));
    AQ_TRY(like(dz, z));
    AQ_TRY(like(dv, z));
    AQ_TRY(sequences_ok(z, d_offsets, count));
    if (!floats_ok(d_first) || !floats_ok(d_dlast) || !floats_ok(d_dfirst) || (d_dfirst && (d_dfirst == d_dlast || d_dfirst == d_first)))
        return AQ_EINVAL;
    if (!workspace_ok(d_workspace, workspace_bytes, recurrence_workspace(z->rows, count, z->cols))) return AQ_EINVAL;
    if (count == 0) return AQ_OK;
    return launch_recurrence_backward(*dy, d_dlast, *z, *v, *y, d_offsets, count, d_starts, d_first, *dz, *dv, d_dfirst, (float*)d_workspace,
                                      as_stream(stream));
}

extern "C" aq_status aq_recurrence_step(const aq_matrix* z, const aq_matrix* v, const uint8_t* d_starts, float* d_state, const aq_matrix* y,
                                        void* stream) {
    AQ_TRY(matrix_ok(z));
    AQ_TRY(like(v, z));
    if (y) AQ_TRY(like(y, z));
    if (!floats_ok(d_state) || (!d_state && z->rows > 0)) return AQ_EINVAL;
    return z->rows == 0 ? AQ_OK : launch_recurrence_step(*z, *v, d_starts, d_state, y, as_stream(stream));
}

// ---- the optimizer

namespace {

constexpr int64_t kMostTensors = 1 << 20;

bool moments_ok(const aq_learned& t) {
    if (t.moment_bits != 8 && t.moment_bits != 32) return false;
    if (t.n == 0) return true;
    if (!t.d_m || !t.d_v) return false;
    if (t.moment_bits == 8) return t.d_m_scales && t.d_v_scales && !((uintptr_t)t.d_m & 15) && !((uintptr_t)t.d_v & 15);
    return floats_ok(t.d_m) && floats_ok(t.d_v);
}
template <class Each>
aq_status tensors_ok(const aq_learned* t, int64_t count, Each&& each) {
    if (count < 0 || (!t && count > 0)) return AQ_EINVAL;
    if (count > kMostTensors) return AQ_ESHAPE;
    for (int64_t i = 0; i < count; ++i)
        if (t[i].n < 0 || !each(t[i])) return AQ_EINVAL;
    for (int64_t i = 0; i < count; ++i)
        if (t[i].n > kMostValues) return AQ_ESHAPE;
    return AQ_OK;
}
bool gradient_ok(const aq_learned& t) {
    if (t.g_dtype != AQ_F32 && t.g_dtype != AQ_F16 && t.g_dtype != AQ_BF16) return false;
    return (t.n == 0 || t.d_g) && (uintptr_t)t.d_g % dtype_bytes(t.g_dtype) == 0;
}

}  // namespace

extern "C" aq_status aq_adamw_step(const aq_learned* tensors, int64_t count, const aq_adamw* how, void* stream) {
    AQ_TRY(tensors_ok(tensors, count, [](const aq_learned& t) {
        if (!gradient_ok(t) || !moments_ok(t) || (t.n > 0 && !t.d_w) || !floats_ok(t.d_w)) return false;
        return !t.d_copy || ((t.copy_dtype == AQ_F16 || t.copy_dtype == AQ_BF16) && ((uintptr_t)t.d_copy & 1) == 0);
    }));
    if (!how || !(how->beta1 >= 0.0 && how->beta1 < 1.0) || !(how->beta2 >= 0.0 && how->beta2 < 1.0) || !(how->eps >= 0.0) ||
        !(how->weight_decay >= 0.0) || !(how->max_norm > 0.0))
        return AQ_EINVAL;
    if (!how->d_lr && !(how->lr >= 0.0)) return AQ_EINVAL;
    if (!how->d_step && how->step < 1) return AQ_EINVAL;
    if (!floats_ok(how->d_lr) || !floats_ok(how->d_norm) || ((uintptr_t)how->d_step & 7)) return AQ_EINVAL;
    return launch_adamw(tensors, count, *how, as_stream(stream));
}

extern "C" aq_status aq_grad_norm_workspace(const aq_learned* tensors, int64_t count, uint64_t* bytes) {
    AQ_TRY(tensors_ok(tensors, count, [](const aq_learned&) { return true; }));
    if (!bytes) return AQ_EINVAL;
    *bytes = (uint64_t)grad_norm_workspace(tensors, count);
    return AQ_OK;
}

extern "C" aq_status aq_grad_norm(const aq_learned* tensors, int64_t count, float* d_norm, void* d_workspace, uint64_t workspace_bytes, void* stream) {
    AQ_TRY(tensors_ok(tensors, count, gradient_ok));
    if (!d_norm || !floats_ok(d_norm) || !workspace_ok(d_workspace, workspace_bytes, grad_norm_workspace(tensors, count))) return AQ_EINVAL;
    return launch_grad_norm(tensors, count, d_norm, d_workspace, as_stream(stream));
}

extern "C" aq_status aq_moments_convert(const aq_learned* from, const aq_learned* to, int64_t count, void* stream) {
    AQ_TRY(tensors_ok(from, count, moments_ok));
    AQ_TRY(tensors_ok(to, count, moments_ok));
    for (int64_t i = 0; i < count; ++i)
        if (from[i].n != to[i].n) return AQ_ESHAPE;
    return launch_moments_convert(from, to, count, as_stream(stream));
}
