#include "lif_packed_launch.h"

namespace lif {
void launch_product_f16(const ProductArgs& a, bool zeros, hipStream_t s) { launch_product_as<_Float16>(a, zeros, s); }
}  // namespace lif
