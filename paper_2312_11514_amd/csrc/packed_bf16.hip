#include "lif_packed_launch.h"

namespace lif {
void launch_product_bf16(const ProductArgs& a, bool zeros, hipStream_t s) { launch_product_as<__bf16>(a, zeros, s); }
}  // namespace lif
