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

}  // namespace aq
