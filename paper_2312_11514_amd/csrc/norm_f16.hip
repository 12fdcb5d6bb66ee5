#include "lif_norm.h"

namespace lif {
void launch_add_norm_f16(const NormArgs& a, hipStream_t s) { launch_add_norm_as<_Float16>(a, s); }
}  // namespace lif
