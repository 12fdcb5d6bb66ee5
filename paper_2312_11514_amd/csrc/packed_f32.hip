#include "lif_packed_launch.h"

namespace lif {
bool launch_product_f32(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s) { return launch_product_as<float>(a, f, zeros, s); }
}  // namespace lif
