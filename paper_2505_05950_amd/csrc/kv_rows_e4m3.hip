// Instances of the rows kernel on e4m3 codes.
#include "kv_rows_launch.h"

namespace floe {
hipError_t launch_kv_rows_e4m3(const KvAttnArgs& a, int mt, hipStream_t st) { return kv_rows_dispatch<kKvE4m3>(a, mt, st); }
}  // namespace floe
