#include "lif_kv_attend.h"

namespace lif {
void launch_attend_f16(const KvView& kv, const AttendArgs& a, int dim_pad, int tiles, int groups, hipStream_t s) {
    launch_attend_as<_Float16>(kv, a, dim_pad, tiles, groups, s);
}
}  // namespace lif
