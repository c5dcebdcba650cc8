// The gated layer's products: the gradient of its input.
#include "gated.hpp"

namespace aq {

aq_status launch_gated_input_product(int type, int s, bool part, const Product& p, const Outputs& out, int slices, hipStream_t st) {
    return launch_gated_product<kInputGrad>(type, s, part, p, out, 0, slices, st);
}

}  // namespace aq
