// Host side of the prompt kernel: one instance per head size and code format.
#pragma once

#include "kv_prompt.h"

namespace floe {

template <int FMT, int D>
hipError_t kv_prompt_instance(const KvAttnArgs& a, hipStream_t st) {
    constexpr int kWaves = kv_prompt_waves(D);
    const dim3 grid(a.prompt_tiles * a.s.n_seqs * a.c.heads, a.prompt_chunks);
    kv_prompt_kernel<D, FMT, kWaves><<<grid, dim3(64 * kWaves), 0, st>>>(a);
    return hipGetLastError();
}
template <int FMT>
hipError_t kv_prompt_dispatch(const KvAttnArgs& a, hipStream_t st) {
    switch (a.c.dim) {
        case 64: return kv_prompt_instance<FMT, 64>(a, st);
        case 128: return kv_prompt_instance<FMT, 128>(a, st);
        case 192: return kv_prompt_instance<FMT, 192>(a, st);
        default: return kv_prompt_instance<FMT, 256>(a, st);
    }
}

}  // namespace floe
