// Host side of the rows kernel: one instance per head size, code format and tiles of sixteen rows.
#pragma once

#include "kv_rows.h"

namespace floe {

template <int FMT, int D, int MT>
hipError_t kv_rows_instance(const KvAttnArgs& a, int workgroups, int rows, hipStream_t st) {
    const dim3 wg(64 * kRowsWaves);
    if (workgroups == 0) {
        const int tiles = (rows * a.group + 16 * MT - 1) / (16 * MT);
        kv_rows_kernel<D, FMT, MT, true><<<dim3(a.c.heads * tiles, a.s.n_seqs), wg, 0, st>>>(a, 0);
    } else {
        kv_rows_kernel<D, FMT, MT, false><<<dim3(workgroups), wg, 0, st>>>(a, kKvMinShare);
    }
    return hipGetLastError();
}
template <int FMT, int D>
hipError_t kv_rows_tiles(const KvAttnArgs& a, int mt, int workgroups, int rows, hipStream_t st) {
    if constexpr (kv_rows_most_tiles(D) >= 4) {
        if (mt == 4) return kv_rows_instance<FMT, D, 4>(a, workgroups, rows, st);
    }
    if constexpr (kv_rows_most_tiles(D) >= 2) {
        if (mt == 2) return kv_rows_instance<FMT, D, 2>(a, workgroups, rows, st);
    }
    return kv_rows_instance<FMT, D, 1>(a, workgroups, rows, st);
}
template <int FMT>
hipError_t kv_rows_dispatch(const KvAttnArgs& a, int mt, int workgroups, int rows, hipStream_t st) {
    switch (a.c.dim) {
        case 64: return kv_rows_tiles<FMT, 64>(a, mt, workgroups, rows, st);
        case 128: return kv_rows_tiles<FMT, 128>(a, mt, workgroups, rows, st);
        case 192: return kv_rows_tiles<FMT, 192>(a, mt, workgroups, rows, st);
        default: return kv_rows_tiles<FMT, 256>(a, mt, workgroups, rows, st);
    }
}

}  // namespace floe
