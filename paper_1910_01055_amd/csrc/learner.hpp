// Host-side launchers of the learner's operators (internal to the library).  Arguments are checked by the entry points.
#pragma once
#include "kernels.hpp"

namespace aq {

// calls go(T()) with the element type of `dtype`
template <class Go>
inline aq_status with_dtype(int32_t dtype, Go&& go) {
    if (dtype == AQ_F32) return go(float());
    if (dtype == AQ_F16) return go(_Float16());
    return go(__bf16());
}
inline size_t dtype_bytes(int32_t dtype) { return dtype == AQ_F32 ? 4 : 2; }
inline int64_t blocks32(int64_t cols) { return (cols + 31) / 32; }

// Lets a kernel have `bytes` of dynamic LDS, once (Key...: what tells it from the others).
template <class... Key>
inline bool allow_lds(const void* kernel, int bytes) {
    static std::atomic<bool> set{false};
    if (bytes > 64 * 1024 && !set) {
        if (hip_failed(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes))) return false;
        set = true;
    }
    return true;
}

// scratch of the caller's: enough, and where 16-byte accesses may begin
inline bool workspace_ok(const void* ws, uint64_t have, int64_t need) {
    return (uint64_t)need <= have && (need == 0 || ws) && ((uintptr_t)ws & 15) == 0;
}

// ---- layernorm.hip
aq_status launch_layernorm_forward(const aq_matrix& x, const float* gamma, const float* beta, float eps, const aq_matrix& y,
                                   float* mean, float* rstd, const aq_ckpt8* kept, hipStream_t st);
int64_t layernorm_backward_workspace(int64_t rows, int64_t cols);
aq_status launch_layernorm_backward(const aq_matrix& dy, const aq_matrix* x, const aq_ckpt8* kept, const float* gamma, const float* mean,
                                    const float* rstd, const aq_matrix& dx, float* dgamma, float* dbeta, float* ws, hipStream_t st);
// ---- blocks32.hip
aq_status launch_ckpt8_pack(const aq_matrix& x, const aq_ckpt8& kept, hipStream_t st);
aq_status launch_ckpt8_unpack(const aq_ckpt8& kept, const aq_matrix& x, hipStream_t st);
aq_status launch_mx4_quantize(const aq_matrix& x, const aq_mx4& q, hipStream_t st);
aq_status launch_mx4_dequantize(const aq_mx4& q, const aq_matrix& x, hipStream_t st);
// ---- mx4_product.hip
int64_t mx4_linear_workspace(int64_t rows, int64_t n, int64_t k);
aq_status launch_mx4_linear(const aq_matrix& x, const aq_mx4& w, const float* bias, const aq_matrix& y, void* ws, hipStream_t st);
aq_status launch_mx4_matmul(const aq_mx4& x, const aq_mx4& w, const float* bias, const aq_matrix& y, hipStream_t st);
// ---- grad_product.hip
int64_t weight_grad_workspace(int64_t rows, int64_t n, int64_t k);
aq_status launch_weight_grad(const aq_matrix& dy, const aq_ckpt8& kept, const aq_matrix& dw, float* db, void* ws, uint64_t ws_bytes,
                             hipStream_t st);
int64_t input_grad_workspace(int64_t rows, int64_t n, int64_t k);
aq_status launch_input_grad(const aq_matrix& dy, const aq_mx4& w, const aq_matrix& dx, void* ws, uint64_t ws_bytes, hipStream_t st);
// ---- gated.hip
int64_t gated_forward_workspace(int64_t rows, int64_t n, int64_t k, int32_t dtype);
int64_t gated_backward_workspace(int64_t rows, int64_t n, int64_t k, int32_t dtype);
aq_status launch_gated_forward(const aq_matrix& x, const aq_matrix& wg, const aq_matrix& wu, int act, const aq_matrix& y, const aq_matrix* gate,
                               const aq_matrix* up, void* ws, hipStream_t st);
aq_status launch_gated_backward(const aq_matrix& dy, const aq_matrix& x, const aq_matrix& wg, const aq_matrix& wu, const aq_matrix& gate,
                                const aq_matrix& up, int act, const aq_matrix* dx, const aq_matrix* dwg, const aq_matrix* dwu, void* ws,
                                hipStream_t st);
// ---- recurrence.hip
int64_t recurrence_workspace(int64_t rows, int64_t count, int64_t cols);
aq_status launch_recurrence_forward(const aq_matrix& z, const aq_matrix& v, const int32_t* offsets, int64_t count, const uint8_t* starts,
                                    const float* first, const aq_matrix& y, float* last, float* ws, hipStream_t st);
aq_status launch_recurrence_backward(const aq_matrix& dy, const float* dlast, const aq_matrix& z, const aq_matrix& v, const aq_matrix& y,
                                     const int32_t* offsets, int64_t count, const uint8_t* starts, const float* first, const aq_matrix& dz,
                                     const aq_matrix& dv, float* dfirst, float* ws, hipStream_t st);
aq_status launch_recurrence_step(const aq_matrix& z, const aq_matrix& v, const uint8_t* starts, float* state, const aq_matrix* y, hipStream_t st);
// ---- adamw.hip
constexpr int64_t kMostValues = 1LL << 34;  // of a tensor
int64_t grad_norm_workspace(const aq_learned* t, int64_t count);
aq_status launch_grad_norm(const aq_learned* t, int64_t count, float* norm, void* ws, hipStream_t st);
aq_status launch_adamw(const aq_learned* t, int64_t count, const aq_adamw& h, hipStream_t st);
aq_status launch_moments_convert(const aq_learned* from, const aq_learned* to, int64_t count, hipStream_t st);

}  // namespace aq
