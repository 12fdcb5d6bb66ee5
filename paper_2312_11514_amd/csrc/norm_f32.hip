#include "lif_norm.h"

namespace lif {
void launch_add_norm_f32(const NormArgs& a, hipStream_t s) { launch_add_norm_as<float>(a, s); }
}  // namespace lif
