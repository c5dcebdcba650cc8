// The gated layer's products: its forward pass.
#include "gated.hpp"

namespace aq {

aq_status launch_gated_forward_product(int type, int s, bool part, const Product& p, const Outputs& out, int act, int slices, hipStream_t st) {
    return launch_gated_product<kForward>(type, s, part, p, out, act, slices, st);
}

}  // namespace aq
