#include "lif_kv_attend.h"

namespace lif {
bool launch_attend_f32_1(const AttendArgs& a, int groups, int waves, hipStream_t s) { return launch_attend_tiles<float, 1>(a, groups, waves, s); }
}  // namespace lif
