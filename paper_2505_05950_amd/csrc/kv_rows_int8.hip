// Instances of the rows kernel on int8 codes.
#include "kv_rows_launch.h"

namespace floe {
hipError_t launch_kv_rows_int8(const KvAttnArgs& a, int mt, hipStream_t st) { return kv_rows_dispatch<kKvInt8, false>(a, mt, st); }
}  // namespace floe
