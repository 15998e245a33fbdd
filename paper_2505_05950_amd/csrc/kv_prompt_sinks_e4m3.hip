// Instances of the prompt kernel with first tokens beside a window, on e4m3 codes.
#include "kv_prompt_launch.h"

namespace floe {
hipError_t launch_kv_prompt_sinks_e4m3(const KvAttnArgs& a, hipStream_t st) { return kv_prompt_dispatch<kKvE4m3, true>(a, st); }
}  // namespace floe
