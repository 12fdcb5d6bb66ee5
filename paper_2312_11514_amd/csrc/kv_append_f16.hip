#include "lif_kv_append.h"

namespace lif {
void launch_append_f16(const KvView& kv, const AppendArgs& a, bool interleaved, hipStream_t s) { launch_append_as<_Float16>(kv, a, interleaved, s); }
}  // namespace lif
