// Beam search's selection over beams and vocabulary.
//
// Mathematics: c(row, token) = score[row] + (x - m) - log sum exp(x - m); the best `take` of a group of rows.  Within a row c orders as x
// does, so one pass over a row's logits yields all that a group needs of it: m, the sum, and the row's best `take` by (x, token).
//
// What bounds it: the bytes of the logits.  beam_rows_kernel: a workgroup takes a slice of a row, its four waves the slice's tiles in turn,
// without a barrier: each lane keeps a running maximum and sum, each wave a threshold that at least `take` of the values that it has seen
// reach.  What reaches the threshold goes to a list in LDS; where that is full, it is cut to its best `take` and the threshold rises.  The
// first threshold is the take-th largest of the 64 lanes' maxima in the wave's first tile (why `take` is at most 64).
// beam_groups_kernel: a workgroup per group joins the slices' sums and finds the best of their lists by the same two steps.
#include "beam.h"

namespace floe {

namespace {

constexpr int kList = 256;  // places of a wave's list
constexpr int kTileLoads = 4;  // of sixteen bytes per lane and tile

// x as an integer that orders alike, and with the token behind it: larger is better, 0 is none (x is finite)
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) {
    return __builtin_bit_cast(float, order ^ ((order & 0x80000000u) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint64_t entry_of(float x, int token) { return ((uint64_t)order_of(x) << 32) | (0xffffffffu - (uint32_t)token); }
__device__ __forceinline__ int token_of(uint64_t e) { return (int)(0xffffffffu - (uint32_t)e); }

// The largest T that at least `take` of the wave's 64 N values reach (0 if there are fewer); bits below `low` are left zero.
template <int N, class U>
__device__ __forceinline__ U wave_kth(const U (&v)[N], int take, int low) {
    U t = 0;
    for (int bit = 8 * (int)sizeof(U) - 1; bit >= low; --bit) {
        const U c = t | ((U)1 << bit);
        int n = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) n += __popcll(__ballot(v[j] >= c));
        if (n >= take) t = c;
    }
    return t;
}
// Cuts `n` entries of a wave's list to the best `take`, which come to its front; returns how many there are.  `least`: the order of the
// last of them, where there are as many.
__device__ __forceinline__ int cut_list(uint64_t* list, int n, int take, uint32_t& least) {
    const int lane = threadIdx.x & 63;
    if (n < take) return n;
    uint64_t v[kList / kWave];
#pragma unroll
    for (int j = 0; j < kList / kWave; ++j) v[j] = j * kWave + lane < n ? list[j * kWave + lane] : 0;
    uint32_t hi[kList / kWave];
#pragma unroll
    for (int j = 0; j < kList / kWave; ++j) hi[j] = (uint32_t)(v[j] >> 32);
    least = wave_kth(hi, take, 0);
    uint64_t bound = (uint64_t)least << 32;
    int reach = 0;
#pragma unroll
    for (int j = 0; j < kList / kWave; ++j) reach += __popcll(__ballot(v[j] >= bound));
    if (reach > take) bound = wave_kth(v, take, 0);  // (several of the same value: the lower tokens)
    int at = 0;
#pragma unroll
    for (int j = 0; j < kList / kWave; ++j) {
        const bool keep = v[j] >= bound && v[j] != 0;
        const uint64_t mask = __ballot(keep);
        if (keep) list[at + __popcll(mask & ((1ull << lane) - 1))] = v[j];
        at += __popcll(mask);
    }
    return at;
}

template <int DTYPE>
constexpr int kElements = DTYPE == 2 ? 4 : 8;  // of sixteen bytes

template <int DTYPE>
__device__ __forceinline__ float logit(const void* row, int i) {
    if constexpr (DTYPE == 2) return gloadf(static_cast<const float*>(row) + i);
    else return from16<DTYPE == 1>(gload2(static_cast<const uint16_t*>(row) + i));
}
__device__ __forceinline__ uint4 gload16_any(const void* p) {  // from any multiple of two bytes
    typedef u32x4 u32x4_2 __attribute__((aligned(2)));
    const u32x4 q = *(const FLOE_GLOBAL u32x4_2*)p;
    return make_uint4(q.x, q.y, q.z, q.w);
}
template <int DTYPE>
struct BeamTile {
    uint4 raw[kTileLoads];
};
template <int DTYPE>
__device__ __forceinline__ void unpack(uint4 q, float* x) {
    if constexpr (DTYPE == 2) {
        x[0] = __builtin_bit_cast(float, q.x), x[1] = __builtin_bit_cast(float, q.y);
        x[2] = __builtin_bit_cast(float, q.z), x[3] = __builtin_bit_cast(float, q.w);
    } else {
        unpack8<DTYPE == 1>(q, x);
    }
}

template <int DTYPE>
__global__ __launch_bounds__(kBeamThreads) void beam_rows_kernel(BeamArgs a) {
    constexpr int E = kElements<DTYPE>, kTile = kTileLoads * kWave * E, kValues = kTileLoads * E;
    constexpr float kLargest = 3.4028234663852886e38f, kInf = __builtin_inff();
    __shared__ uint64_t lists[kBeamWaves][kList];
    __shared__ float wave_sums[kBeamWaves][2];
    __shared__ int kept[kBeamWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x / a.slices, part = blockIdx.x - row * a.slices;
    if (!(a.score[row] > -kInf) || (a.done && a.done[row])) return;  // (the groups' kernel does not look at such a row either)
    constexpr int kSize = DTYPE == 2 ? 4 : 2;
    const unsigned char* logits = static_cast<const unsigned char*>(a.logits) + row * a.stride * kSize;
    const int begin = part * a.slice, end = min(a.vocab, begin + a.slice);
    uint64_t* list = lists[wave];
    float top = -kInf;   // of the lane
    double sum = 0.0;    // (tiles are summed in 32 bits, and their sums in 64: chains of eight, however long the row)
    float bar = -kLargest;          // the wave's threshold
    int n = 0;                      // entries of its list
    bool first = true;
    auto load = [&](int t0, BeamTile<DTYPE>& f) {
#pragma unroll
        for (int u = 0; u < kTileLoads; ++u) {
            const int i = t0 + (u * kWave + lane) * E;
            if (i + E <= end) f.raw[u] = gload16_any(logits + (size_t)i * kSize);
        }
    };
    auto take_tile = [&](int t0, const BeamTile<DTYPE>& f) {
        float x[kValues];
#pragma unroll
        for (int u = 0; u < kTileLoads; ++u) {
            const int i = t0 + (u * kWave + lane) * E;
            if (i + E <= end) {
                unpack<DTYPE>(f.raw[u], x + u * E);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) x[u * E + e] = i + e < end ? logit<DTYPE>(logits, i + e) : -kInf;
            }
        }
        float most = -kInf;
#pragma unroll
        for (int j = 0; j < kValues; ++j) {
            x[j] = fminf(fmaxf(x[j], -kInf), kLargest);  // (a NaN becomes -infinity)
            most = fmaxf(most, x[j]);
        }
        const float grown = fmaxf(top, most), base = grown == -kInf ? 0.0f : grown;
        float part[kTileLoads];
#pragma unroll
        for (int u = 0; u < kTileLoads; ++u) {
            part[u] = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) part[u] += __builtin_amdgcn_exp2f((x[u * E + e] - base) * 1.4426950408889634f);
        }
        sum = sum * (double)__builtin_amdgcn_exp2f((top - base) * 1.4426950408889634f) + (double)((part[0] + part[1]) + (part[2] + part[3]));
        top = grown;
        // candidates
        bool raised = first;
        if (first) {
            const uint32_t v[1] = {order_of(most + 0.0f)};
            const uint32_t t = wave_kth(v, a.take, 8);
            bar = t == 0 ? bar : fmaxf(bar, value_of(t));
            first = false;
        }
        if (__ballot(most >= bar) == 0) return;
        uint32_t least = 0;
#pragma unroll
        for (int j = 0; j < kValues; ++j) {
            const uint64_t mask = __ballot(x[j] >= bar);
            if (mask == 0) continue;
            if (n + __popcll(mask) > kList) {
                n = cut_list(list, n, a.take, least);
                // (of this tile lower tokens may still come with the same value)
                bar = fmaxf(bar, value_of(least));
                raised = true;
            }
            const uint64_t now = __ballot(x[j] >= bar);
            if (x[j] >= bar) list[n + __popcll(now & ((1ull << lane) - 1))] = entry_of(x[j] + 0.0f, t0 + ((j / E) * kWave + lane) * E + j % E);
            n += __popcll(now);
        }
        if (raised && n >= a.take) bar = value_of(order_of(bar) + 1);  // tokens of later tiles lose to those that have the same value
    };
    const int stride = kBeamWaves * kTile;
    BeamTile<DTYPE> f0, f1;
    int t0 = begin + wave * kTile;
    load(t0, f0);
    for (; t0 < end; t0 += 2 * stride) {
        load(t0 + stride, f1);
        take_tile(t0, f0);
        if (t0 + stride >= end) break;
        load(t0 + 2 * stride, f0);
        take_tile(t0 + stride, f1);
    }
    // ---- the four waves meet
    uint32_t least = 0;
    n = cut_list(list, n, a.take, least);
    float all = top;
#pragma unroll
    for (int step = 32; step; step >>= 1) all = fmaxf(all, __shfl_xor(all, step));
    sum *= (double)__builtin_amdgcn_exp2f((top - (all == -kInf ? 0.0f : all)) * 1.4426950408889634f);
#pragma unroll
    for (int step = 32; step; step >>= 1) sum += __shfl_xor(sum, step);
    if (lane == 0) {
        wave_sums[wave][0] = all;
        wave_sums[wave][1] = (float)sum;
        kept[wave] = n;
    }
    __syncthreads();
    if (wave != 0) return;
    float m = -kInf, s = 0.0f;
#pragma unroll
    for (int k = 0; k < kBeamWaves; ++k) m = fmaxf(m, wave_sums[k][0]);
#pragma unroll
    for (int k = 0; k < kBeamWaves; ++k) s += wave_sums[k][1] * __builtin_amdgcn_exp2f((wave_sums[k][0] - (m == -kInf ? 0.0f : m)) * 1.4426950408889634f);
    for (int k = 1; k < kBeamWaves; ++k) {
        if (lane < kept[k]) list[n + lane] = lists[k][lane];
        n += kept[k];
    }
    __builtin_amdgcn_wave_barrier();
    n = cut_list(list, n, a.take, least);
    if (lane == 0) {
        a.sums[2 * blockIdx.x] = m;
        a.sums[2 * blockIdx.x + 1] = s;
    }
    if (lane < a.take) a.best[(size_t)blockIdx.x * a.take + lane] = lane < n ? list[lane] : 0;
}

// A workgroup per group.
constexpr int kGroupThreads = 1024, kGroupWaves = kGroupThreads / kWave;
constexpr int kGroupList = 1024;  // candidates that reach the group's threshold and are ordered at a time
struct Candidate {
    double c;
    uint64_t entry;
    int row;
};
__device__ __forceinline__ bool before(double c, int row, uint64_t e, double c2, int row2, uint64_t e2) {
    return c > c2 || (c == c2 && (row < row2 || (row == row2 && e > e2)));
}
__global__ __launch_bounds__(kGroupThreads) void beam_groups_kernel(BeamArgs a) {
    constexpr float kInf = __builtin_inff();
    __shared__ double log_sum[kBeamRows];
    __shared__ float row_top[kBeamRows], row_score[kBeamRows];
    __shared__ uint8_t row_kind[kBeamRows];  // 0: offers nothing, 1: tokens, 2: its end
    __shared__ uint32_t lane_top[kGroupWaves][kWave];
    __shared__ double list_c[kGroupList];
    __shared__ uint64_t list_e[kGroupList];
    __shared__ int16_t list_row[kGroupList];
    __shared__ uint32_t bar_order;
    __shared__ int listed;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, group = blockIdx.x;
    for (int r = tid; r < a.beams; r += kGroupThreads) {
        const int row = group * a.beams + r;
        const float score = a.score[row];
        const bool alive = score > -kInf, ended = a.done && a.done[row];
        float m = -kInf;
        double s = 0.0;
        if (alive && !ended) {
            const float* sums = a.sums + (size_t)row * a.slices * 2;
            for (int k = 0; k < a.slices; ++k) m = fmaxf(m, sums[2 * k]);
            if (m > -kInf)
                for (int k = 0; k < a.slices; ++k)
                    if (sums[2 * k] > -kInf) s += (double)sums[2 * k + 1] * exp((double)sums[2 * k] - (double)m);
        }
        row_top[r] = m;
        log_sum[r] = s > 0.0 ? log(s) : 0.0;
        row_score[r] = score;
        row_kind[r] = !alive ? 0 : ended ? 2 : m > -kInf ? 1 : 0;
    }
    __syncthreads();
    const int per_row = a.slices * a.take, all = a.beams * per_row;
    // the id-th candidate of the group
    auto candidate = [&](int id) {
        Candidate x;
        x.row = id / per_row;
        const int k = id - x.row * per_row, kind = row_kind[x.row];
        x.c = -(double)kInf;
        x.entry = 0;
        if (kind == 1) {
            x.entry = a.best[((size_t)(group * a.beams + x.row) * a.slices) * a.take + k];
            if (x.entry) x.c = (double)row_score[x.row] + (((double)value_of((uint32_t)(x.entry >> 32)) - (double)row_top[x.row]) - log_sum[x.row]);
        } else if (kind == 2 && k == 0) {
            x.entry = entry_of(0.0f, a.eos);
            x.c = (double)row_score[x.row];
        }
        return x;
    };
    // a threshold that at least `take` candidates reach: the take-th largest of 64 maxima, in binary32 rounded down
    float most = -kInf;
    for (int id = tid; id < all; id += kGroupThreads) {
        const double c = candidate(id).c;
        const float f = (float)c;
        most = fmaxf(most, (double)f > c ? value_of(order_of(f) - 1) : f);
    }
    lane_top[wave][lane] = order_of(most);
    if (tid == 0) listed = 0;
    __syncthreads();
    if (wave == 0) {
        uint32_t v[1] = {0};
        for (int k = 0; k < kGroupWaves; ++k) v[0] = max(v[0], lane_top[k][lane]);
        const uint32_t t = wave_kth(v, a.take, 0);
        if (lane == 0) bar_order = t;
    }
    __syncthreads();
    const float bar = value_of(bar_order);
    for (int id = tid; id < all; id += kGroupThreads) {
        const Candidate x = candidate(id);
        if (x.entry == 0 || !(x.c >= (double)bar)) continue;
        const int at = atomicAdd(&listed, 1);
        if (at < kGroupList) list_c[at] = x.c, list_e[at] = x.entry, list_row[at] = (int16_t)x.row;
    }
    __syncthreads();
    const int n = min(listed, kGroupList);
    const size_t out = (size_t)group * a.take;
    auto write = [&](int rank, double c, int row, uint64_t e) {
        const int token = token_of(e);
        a.score_out[out + rank] = (float)c;
        a.parent[out + rank] = group * a.beams + row;
        a.token[out + rank] = token;
        if (a.done_out) a.done_out[out + rank] = token == a.eos || row_kind[row] == 2;
    };
    if (listed <= kGroupList) {
        for (int i = tid; i < n; i += kGroupThreads) {
            const double c = list_c[i];
            const uint64_t e = list_e[i];
            const int row = list_row[i];
            int rank = 0;
            for (int k = 0; k < n; ++k) rank += before(list_c[k], list_row[k], list_e[k], c, row, e);
            if (rank < a.take) write(rank, c, row, e);
        }
    } else {
        // more than the list holds: every candidate that reaches the threshold against all others
        for (int id = tid; id < all; id += kGroupThreads) {
            const Candidate x = candidate(id);
            if (x.entry == 0 || !(x.c >= (double)bar)) continue;
            int rank = 0;
            for (int k = 0; k < all && rank < a.take; ++k) {
                const Candidate y = candidate(k);
                rank += y.entry != 0 && before(y.c, y.row, y.entry, x.c, x.row, x.entry);
            }
            if (rank < a.take) write(rank, x.c, x.row, x.entry);
        }
    }
    if (tid >= listed && tid < a.take) {
        a.score_out[out + tid] = -kInf;
        a.parent[out + tid] = -1;
        a.token[out + tid] = -1;
        if (a.done_out) a.done_out[out + tid] = 0;
    }
}

}  // namespace

// A slice is a multiple of what a workgroup's four waves take at a time, as large as leaves every compute unit four workgroups.
BeamCut beam_cut(int rows, int vocab, int dtype) {
    const int step = kBeamWaves * kTileLoads * kWave * (dtype == 2 ? 4 : 8), steps = (vocab + step - 1) / step;
    int64_t slices = rows > 0 ? (4ll * num_cus() + rows - 1) / rows : 1;
    if (slices > steps) slices = steps;
    const int per = (int)((steps + slices - 1) / slices);
    return BeamCut{(steps + per - 1) / per, per * step};
}

hipError_t launch_beam_rows(const BeamArgs& a, int dtype, hipStream_t st) {
    const dim3 grid(a.groups * a.beams * a.slices), wg(kBeamThreads);
    if (dtype == 0) beam_rows_kernel<0><<<grid, wg, 0, st>>>(a);
    else if (dtype == 1) beam_rows_kernel<1><<<grid, wg, 0, st>>>(a);
    else beam_rows_kernel<2><<<grid, wg, 0, st>>>(a);
    return hipGetLastError();
}
hipError_t launch_beam_groups(const BeamArgs& a, hipStream_t st) {
    beam_groups_kernel<<<dim3(a.groups), dim3(kGroupThreads), 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace floe
