#include "lif_packed_launch.h"

namespace lif {
void launch_product_i8_groups(const ProductArgs& a, bool zeros, hipStream_t s) { launch_product_as<ByGroup>(a, zeros, s); }
}  // namespace lif
