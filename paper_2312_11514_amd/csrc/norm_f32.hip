#include "lif_norm.h"

namespace lif {
void launch_add_norm_f32(const NormArgs& a, int rows, hipStream_t s) { launch_add_norm_as<float>(a, rows, s); }
}  // namespace lif
