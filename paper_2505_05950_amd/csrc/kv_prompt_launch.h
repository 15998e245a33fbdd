// Host side of the prompt kernel: one instance per head size, code format and number of waves, with and without first tokens beside a window.
#pragma once

#include "kv_prompt.h"

namespace floe {

template <int FMT, bool SINKS, int D, int NW>
hipError_t kv_prompt_instance(const KvAttnArgs& a, hipStream_t st) {
    kv_prompt_kernel<D, FMT, NW, SINKS><<<dim3(a.prompt_tiles * a.s.n_seqs * a.c.heads, a.prompt_chunks), dim3(64 * NW), 0, st>>>(a);
    return hipGetLastError();
}
template <int FMT, bool SINKS>
hipError_t kv_prompt_dispatch(const KvAttnArgs& a, hipStream_t st) {
    switch (a.c.dim) {
        case 64: return kv_prompt_instance<FMT, SINKS, 64, 4>(a, st);
        case 128: return a.prompt_waves == 4 ? kv_prompt_instance<FMT, SINKS, 128, 4>(a, st) : kv_prompt_instance<FMT, SINKS, 128, 8>(a, st);
        case 192: return a.prompt_waves == 4 ? kv_prompt_instance<FMT, SINKS, 192, 4>(a, st) : kv_prompt_instance<FMT, SINKS, 192, 8>(a, st);
        default: return a.prompt_waves == 4 ? kv_prompt_instance<FMT, SINKS, 256, 4>(a, st) : kv_prompt_instance<FMT, SINKS, 256, 8>(a, st);
    }
}

}  // namespace floe
