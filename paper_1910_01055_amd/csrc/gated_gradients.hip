// The gated layer's products: both gradients in one launch.
#include "gated.hpp"

namespace aq {

aq_status launch_gated_gradients(int type, int s, const Product& dx, const Outputs& out_dx, int slices_dx, const Product& dw, const Outputs& out_dw, int slices_dw,
                                 hipStream_t st) {
    auto sized = [&](auto h, auto t, auto size, auto planes) {
        using H = decltype(h);
        using T = decltype(t);
        constexpr int S = decltype(size)::value, P = decltype(planes)::value, kLds = gated_lds(S, kInputGrad, P);
        static_assert(kLds <= kMostLds && kLds == gated_lds(S, kWeightGrad, P), "");
        auto* const k = k_gated_gradients<H, T, S, P>;
        const int64_t inputs = (int64_t)dx.tiles_m * dx.tiles_c * slices_dx, weights = (int64_t)dw.tiles_m * 2 * dw.tiles_c * slices_dw;
        if (!grid_ok(inputs + weights, 2 * S)) return AQ_ESHAPE;
        if (!allow_lds<H, T, decltype(size), decltype(planes)>((const void*)k, kLds)) return AQ_EHIP;
        const bool weights_first = inputs == 0 || (weights != 0 && dw.chunks > dx.chunks);
        k<<<(unsigned)(inputs + weights), 2 * S, kLds, st>>>(dx, out_dx, dw, out_dw, (uint32_t)(weights_first ? weights : inputs), weights_first);
        return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
    };
    constexpr std::integral_constant<int, 64> small{};
    constexpr std::integral_constant<int, 128> large{};
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::integral_constant<int, 3> three{};
    auto typed = [&](auto size) {
        if (type == AQ_F32) return sized(bf16_t(), float(), size, three);
        return type == AQ_F16 ? sized(f16_t(), f16_t(), size, one) : sized(bf16_t(), bf16_t(), size, one);
    };
    return s == 128 ? typed(large) : typed(small);
}

}  // namespace aq
