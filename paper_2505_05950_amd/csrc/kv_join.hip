// Joins what the chunks of the attention kernels left (kv_rows.h, kv_prompt.h).
#include "kv_prompt.h"

namespace floe {

namespace {
template <int D>
hipError_t join_tiles(const KvAttnArgs& a, int mt, int rows, hipStream_t st) {
    const dim3 grid(a.q_heads * rows, a.s.n_seqs), wg(256);
    if constexpr (kv_rows_most_tiles(D) >= 4) {
        if (mt == 4) return kv_join_kernel<D, 4><<<grid, wg, 0, st>>>(a), hipGetLastError();
    }
    if constexpr (kv_rows_most_tiles(D) >= 2) {
        if (mt == 2) return kv_join_kernel<D, 2><<<grid, wg, 0, st>>>(a), hipGetLastError();
    }
    kv_join_kernel<D, 1><<<grid, wg, 0, st>>>(a);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_kv_join(const KvAttnArgs& a, int mt, int rows, hipStream_t st) {
    switch (a.c.dim) {
        case 64: return join_tiles<64>(a, mt, rows, st);
        case 128: return join_tiles<128>(a, mt, rows, st);
        case 192: return join_tiles<192>(a, mt, rows, st);
        default: return join_tiles<256>(a, mt, rows, st);
    }
}

namespace {
template <int D>
hipError_t prompt_join(const KvAttnArgs& a, hipStream_t st) {
    kv_prompt_join_kernel<D><<<dim3(a.q_heads * a.s.max_rows, a.s.n_seqs), dim3(256), 0, st>>>(a);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_kv_prompt_join(const KvAttnArgs& a, hipStream_t st) {
    switch (a.c.dim) {
        case 64: return prompt_join<64>(a, st);
        case 128: return prompt_join<128>(a, st);
        case 192: return prompt_join<192>(a, st);
        default: return prompt_join<256>(a, st);
    }
}

}  // namespace floe
