#include "lif_norm.h"

namespace lif {
void launch_add_norm_bf16(const NormArgs& a, hipStream_t s) { launch_add_norm_as<__bf16>(a, s); }
}  // namespace lif
