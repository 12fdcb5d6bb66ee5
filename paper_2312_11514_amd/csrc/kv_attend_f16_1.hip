#include "lif_kv_attend.h"

namespace lif {
bool launch_attend_f16_1(const AttendArgs& a, int groups, int waves, hipStream_t s) { return launch_attend_tiles<_Float16, 1>(a, groups, waves, s); }
}  // namespace lif
