#include "lif_kv_append.h"

namespace lif {
void launch_append_f32(const KvView& kv, const AppendArgs& a, bool interleaved, hipStream_t s) { launch_append_as<float>(kv, a, interleaved, s); }
}  // namespace lif
