// Instances of the prompt kernel on e4m3 codes.
#include "kv_prompt_launch.h"

namespace floe {
hipError_t launch_kv_prompt_e4m3(const KvAttnArgs& a, hipStream_t st) { return kv_prompt_dispatch<kKvE4m3>(a, st); }
}  // namespace floe
