#include "lif_packed_launch.h"

namespace lif {
void launch_product_i8(const ProductArgs& a, bool zeros, hipStream_t s) { launch_product_as<signed char>(a, zeros, s); }
}  // namespace lif
