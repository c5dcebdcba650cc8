// The gated layer's products: the gradient of its input, on tiles of 256.
#include "gated.hpp"

namespace aq {

aq_status launch_gated_input_product(int type, bool part, const Product& p, const Outputs& out, int slices, hipStream_t st) {
    return launch_gated_large<kInputGrad>(type, part, p, out, 0, slices, st);
}

}  // namespace aq
