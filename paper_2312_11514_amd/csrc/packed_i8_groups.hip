#include "lif_packed_launch.h"

namespace lif {
bool launch_product_i8_groups(const ProductArgs& a, PackedForm f, bool zeros, hipStream_t s) { return launch_product_as<ByGroup>(a, f, zeros, s); }
}  // namespace lif
