#include "lif_norm.h"

namespace lif {
void launch_add_norm_f16(const NormArgs& a, int rows, hipStream_t s) { launch_add_norm_as<_Float16>(a, rows, s); }
}  // namespace lif
