#include "lif_kv_attend.h"

namespace lif {
bool launch_attend_bf16_2(const AttendArgs& a, int groups, int waves, hipStream_t s) { return launch_attend_tiles<__bf16, 2>(a, groups, waves, s); }
}  // namespace lif
