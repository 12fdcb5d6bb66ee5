#include "lif_packed_launch.h"

namespace lif {
bool launch_product_bf16(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s) { return launch_product_as<__bf16>(a, f, zeros, s); }
}  // namespace lif
