// Host side of the prompt kernel: one instance per head size and code format.
#pragma once

#include "kv_prompt.h"

namespace floe {

template <int FMT, int D>
hipError_t kv_prompt_instance(const KvAttnArgs& a, hipStream_t st) {
    constexpr int kWaves = kv_prompt_waves(D), kRows = kv_prompt_rows(D);
    const int tiles = (int)(((int64_t)a.s.max_rows * a.group + kRows - 1) / kRows);
    kv_prompt_kernel<D, FMT, kWaves><<<dim3(tiles * a.s.n_seqs * a.c.heads), dim3(64 * kWaves), 0, st>>>(a, tiles);
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
