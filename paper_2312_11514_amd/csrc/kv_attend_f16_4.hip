#include "lif_kv_attend.h"

namespace lif {
bool launch_attend_f16_4(const AttendArgs& a, int groups, int waves, hipStream_t s) { return launch_attend_tiles<_Float16, 4>(a, groups, waves, s); }
}  // namespace lif
