#include "lif_packed_launch.h"

namespace lif {
bool launch_product_f16(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s) { return launch_product_as<_Float16>(a, f, zeros, s); }
}  // namespace lif
