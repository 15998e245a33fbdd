// Instances of the prompt kernel with first tokens beside a window, on int8 codes.
#include "kv_prompt_launch.h"

namespace floe {
hipError_t launch_kv_prompt_sinks_int8(const KvAttnArgs& a, hipStream_t st) { return kv_prompt_dispatch<kKvInt8, true>(a, st); }
}  // namespace floe
