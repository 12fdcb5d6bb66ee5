#include "lif_packed_launch.h"

namespace lif {
void launch_product_f32(const ProductArgs& a, bool zeros, hipStream_t s) { launch_product_as<float>(a, zeros, s); }
}  // namespace lif
