// The gated layer's products: forward.
#include "gated.hpp"

namespace aq {

aq_status launch_gated_forward_product(int type, int s, bool part, const Product& p, const Outputs& out, int act, int slices, hipStream_t st) {
    auto sized = [&](auto h, auto t, auto parts, auto planes) {
        using H = decltype(h);
        using T = decltype(t);
        constexpr bool kPart = decltype(parts)::value;
        constexpr int P = decltype(planes)::value;
        return s == 128 ? launch_gated_product<H, T, 128, kForward, kPart, P>(p, out, act, slices, st)
                        : launch_gated_product<H, T, 64, kForward, kPart, P>(p, out, act, slices, st);
    };
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::integral_constant<int, 3> three{};
    if (type == AQ_F32) return part ? sized(bf16_t(), float(), std::true_type(), three) : sized(bf16_t(), float(), std::false_type(), three);
    if (s == 256) return launch_gated_large<kForward>(type, part, p, out, act, slices, st);
    if (part) return type == AQ_F16 ? sized(f16_t(), float(), std::true_type(), one) : sized(bf16_t(), float(), std::true_type(), one);
    return type == AQ_F16 ? sized(f16_t(), f16_t(), std::false_type(), one) : sized(bf16_t(), bf16_t(), std::false_type(), one);
}

}  // namespace aq
