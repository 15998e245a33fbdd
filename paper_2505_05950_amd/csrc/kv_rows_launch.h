// Host side of the rows kernel: one instance per head size, code format and tiles of sixteen rows, with and without first tokens
// beside a window.
#pragma once

#include "kv_rows.h"

namespace floe {

template <int FMT, bool SINKS, int D, int MT>
hipError_t kv_rows_instance(const KvAttnArgs& a, hipStream_t st) {
    const dim3 grid(a.s.n_seqs * a.c.heads * a.tiles, a.chunks);
    kv_rows_kernel<D, FMT, MT, SINKS><<<grid, dim3(64 * kRowsWaves), 0, st>>>(a);
    return hipGetLastError();
}
template <int FMT, bool SINKS, int D>
hipError_t kv_rows_tiles(const KvAttnArgs& a, int mt, hipStream_t st) {
    if constexpr (kv_rows_most_tiles(D) >= 4) {
        if (mt == 4) return kv_rows_instance<FMT, SINKS, D, 4>(a, st);
    }
    if constexpr (kv_rows_most_tiles(D) >= 2) {
        if (mt == 2) return kv_rows_instance<FMT, SINKS, D, 2>(a, st);
    }
    return kv_rows_instance<FMT, SINKS, D, 1>(a, st);
}
template <int FMT, bool SINKS>
hipError_t kv_rows_dispatch(const KvAttnArgs& a, int mt, hipStream_t st) {
    switch (a.c.dim) {
        case 64: return kv_rows_tiles<FMT, SINKS, 64>(a, mt, st);
        case 128: return kv_rows_tiles<FMT, SINKS, 128>(a, mt, st);
        case 192: return kv_rows_tiles<FMT, SINKS, 192>(a, mt, st);
        default: return kv_rows_tiles<FMT, SINKS, 256>(a, mt, st);
    }
}

}  // namespace floe
