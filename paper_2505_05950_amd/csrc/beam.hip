// Beam search's selection over beams and vocabulary.
//
// Mathematics: c(row, token) = score[row] + (x - m) - log sum exp(x - m); the best `take` of a group of rows.  Within a row c orders as x
// does, so one pass over a row's logits yields all that a group needs of it: m, the sum, and the row's best `take` by (x, token).
//
// What bounds it: the bytes of the logits, and for few rows the chain load, maximum, threshold, list, join.  beam_rows_kernel: a workgroup takes
// a slice of a row, its four waves the slice's tiles in turn.  Each lane keeps a running maximum and sum; what reaches the workgroup's
// threshold goes to its wave's list in LDS.  The threshold: if each of the waves has seen `quota` values that reach q of its own, with
// quota * waves >= take, then `take` values reach the least of the four q, and what lies below is not among the slice's best.  q is at first
// the quota-th largest of the 64 lanes' maxima in the wave's first tile, later the quota-th best of its list, formed again whenever that has
// grown by some quotas: what passes falls as 1 / tiles then.  A list that would not hold a tile's values is cut to its best `take`, which
// bounds it whatever the values are.
// beam_groups_kernel: a workgroup per group joins the slices' sums, and finds the best of their lists with a threshold formed alike.
#include "beam.h"

namespace floe {

namespace {

constexpr int kList = 256;  // places of a wave's list
constexpr int kListParts = kList / kWave;

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

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = max(x, (uint32_t)dpp_movi<0x128>((int)x));
    x = max(x, (uint32_t)dpp_movi<0x124>((int)x));
    x = max(x, (uint32_t)dpp_movi<0x122>((int)x));
    x = max(x, (uint32_t)dpp_movi<0x121>((int)x));
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __builtin_amdgcn_readfirstlane(max((uint32_t)b[0], (uint32_t)b[1]));
}
__device__ __forceinline__ double halves(uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo); }
template <int CTRL>
__device__ __forceinline__ double dpp_add64(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    return x + halves((uint32_t)dpp_movi<CTRL>((int)(uint32_t)u), (uint32_t)dpp_movi<CTRL>((int)(uint32_t)(u >> 32)));
}
__device__ __forceinline__ double wave_sum64(double x) {
    x = dpp_add64<0x121>(dpp_add64<0x122>(dpp_add64<0x124>(dpp_add64<0x128>(x))));
    uint64_t u = __builtin_bit_cast(uint64_t, x);
    const auto l16 = __builtin_amdgcn_permlane16_swap((uint32_t)u, (uint32_t)u, false, false), h16 = __builtin_amdgcn_permlane16_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    u = __builtin_bit_cast(uint64_t, halves(l16[0], h16[0]) + halves(l16[1], h16[1]));
    const auto l32 = __builtin_amdgcn_permlane32_swap((uint32_t)u, (uint32_t)u, false, false), h32 = __builtin_amdgcn_permlane32_swap((uint32_t)(u >> 32), (uint32_t)(u >> 32), false, false);
    return halves(l32[0], h32[0]) + halves(l32[1], h32[1]);
}
// The largest T that at least `k` of the wave's 64 N values reach (0 if there are fewer), in bits `low` to `high`, with `t` above them
template <int N>
__device__ __forceinline__ uint32_t wave_kth(const uint32_t (&v)[N], int k, int low, int high = 31, uint32_t t = 0) {
#pragma unroll 1  // (unrolled, 53 KB more code: 120 rows of 50257 in bf16 take 8.8 us either way, 512 of 131072 in fp32 57 instead of 59)
    for (int bit = high; bit >= low; --bit) {
        const uint32_t c = t | (1u << bit);
        int n = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) n += __popcll(__ballot(v[j] >= c));
        if (n >= k) t = c;
    }
    return t;
}
// A 16-bit type's values fill the upper bits alone (the lower ones are zeros, of negative values ones), but for what stands for +infinity.
template <int DTYPE>
constexpr int kLowBit = DTYPE == 0 ? 13 : DTYPE == 1 ? 16 : 0;
// The order of the k-th largest value itself
template <int DTYPE, int N>
__device__ __forceinline__ uint32_t wave_kth_order(const uint32_t (&v)[N], int k) {
    const uint32_t t = wave_kth(v, k, kLowBit<DTYPE>);
    if constexpr (DTYPE == 2) return t;
    if (t >= 0xff7f0000u) return wave_kth(v, k, 0, kLowBit<DTYPE> - 1, t);
    return t & 0x80000000u ? t : t | ((1u << kLowBit<DTYPE>) - 1);
}
// Cuts `n` >= take entries of a wave's list to the best `take`, which come to its front.  Returns the order of the least of them.
template <int DTYPE, int N>
__device__ __forceinline__ uint32_t cut_parts(uint64_t* list, int n, int take, int token_bits) {
    const int lane = threadIdx.x & 63;
    uint32_t hi[N], lo[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const uint64_t v = j * kWave + lane < n ? list[j * kWave + lane] : 0;
        hi[j] = (uint32_t)(v >> 32);
        lo[j] = (uint32_t)v;
    }
    const uint32_t t = wave_kth_order<DTYPE>(hi, take);
    int above = 0, reach = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) above += __popcll(__ballot(hi[j] > t)), reach += __popcll(__ballot(hi[j] >= t));
    uint32_t bar = 0;  // of those with that very value, the lower tokens
    if (reach > take) {
        const uint32_t mask = (1u << token_bits) - 1;
        uint32_t tie[N];
#pragma unroll
        for (int j = 0; j < N; ++j) tie[j] = hi[j] == t ? (lo[j] & mask) + 1 : 0;
        bar = wave_kth(tie, take - above, 0, token_bits) - 1 + (0xffffffffu - mask);
    }
    int at = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const bool keep = hi[j] > t || (hi[j] == t && lo[j] >= bar);
        const uint64_t mask = __ballot(keep);
        if (keep) list[at + __popcll(mask & ((1ull << lane) - 1))] = ((uint64_t)hi[j] << 32) | lo[j];
        at += __popcll(mask);
    }
    return t;
}
// Up to 64 entries, one per lane, in order: each lane counts those that are better than its own (a search bit by bit takes three times as long).
__device__ __forceinline__ void sort_few(uint64_t* list, int n) {
    const int lane = threadIdx.x & 63;
    const uint64_t mine = lane < n ? list[lane] : 0;
    const int lo = (int)(uint32_t)mine, hi = (int)(uint32_t)(mine >> 32);
    int rank = 0;
#pragma unroll 1
    for (int k0 = 0; k0 < n; k0 += 4) {  // (lanes behind the last entry hold 0, which is better than none)
#pragma unroll
        for (int k = k0; k < k0 + 4; ++k) {
            const uint64_t e = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, k) << 32) | (uint32_t)__builtin_amdgcn_readlane(lo, k);
            rank += e > mine;
        }
    }
    if (lane < n) list[rank] = mine;
}
// The k-th largest of the wave's 64 values, or a little less: one by one for the first few
__device__ __forceinline__ uint32_t wave_kth_few(uint32_t v, int k) {
    if (k > 4) {
        const uint32_t one[1] = {v};
        return wave_kth(one, k, 12);
    }
    uint32_t m = 0;
#pragma unroll 1
    for (int i = 0; i < k; ++i) {
        m = wave_max(v);
        if ((threadIdx.x & 63) == (unsigned)__builtin_ctzll(__ballot(v == m))) v = 0;
    }
    return m;
}

template <int DTYPE>
constexpr int kElements = DTYPE == 2 ? 4 : 8;  // of sixteen bytes

// exp(d) of d <= 0 to 1e-8; below -100, and for -infinity less itself, that of -100.  exp(d) = 2^n exp(y) with |y| <= log(2) / 2, by its series.
__device__ __forceinline__ double exp_of(double d) {
    const double t = fmax(d, -100.0) * 1.4426950408889634, n = __builtin_rint(t), y = (t - n) * 0.69314718055994531;
    const double p = 1.0 + y * (1.0 + y * (1.0 / 2 + y * (1.0 / 6 + y * (1.0 / 24 + y * (1.0 / 120 + y * (1.0 / 720 + y * (1.0 / 5040)))))));
    return __builtin_amdgcn_ldexp(p, (int)n);
}

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
template <int LOADS>
struct BeamTile {
    uint4 raw[LOADS];
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

// LOADS: of sixteen bytes per lane and tile
template <int DTYPE, int LOADS>
__global__ __launch_bounds__(kBeamThreads) void beam_rows_kernel(BeamArgs a) {
    constexpr int E = kElements<DTYPE>, kTile = LOADS * kWave * E;
    constexpr float kLargest = 3.4028234663852886e38f, kInf = __builtin_inff(), kLog2e = 1.4426950408889634f;
    __shared__ uint64_t lists[kBeamWaves][kList];
    __shared__ BeamSum wave_sums[kBeamWaves];
    __shared__ int kept[kBeamWaves];
    __shared__ uint64_t shares[kBeamWaves / 2];  // q of each wave, as order; of one without a tile the largest
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x / a.slices, part = blockIdx.x - row * a.slices;
    // (-0 becomes 0: candidates are ranked by c as an integer, in which the zeros differ)
    const float score = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, a.score[row] + 0.0f)));
    const bool done = a.done && a.done[row];
    if (!(score > -kInf) || done) {  // nothing of its logits counts
        if (tid == 0) a.sums[blockIdx.x] = BeamSum{-kInf, score, done ? kBeamDone : 0.0};
        return;
    }
    constexpr int kSize = DTYPE == 2 ? 4 : 2;
    const unsigned char* logits = static_cast<const unsigned char*>(a.logits) + row * a.stride * kSize;
    const int begin = part * a.slice, end = min(a.vocab, begin + a.slice), token_bits = 32 - __builtin_clz(a.vocab);
    uint64_t* list = lists[wave];
    float top = -kInf;   // of the lane
    // Terms are exp(x - base) with base <= top <= base + 8: a base that followed every new maximum would have the whole sum multiplied each time,
    // and the factors' roundings would add up over the tiles (2^24 slowly ascending values in one slice: log s off by 5e-5).  One that moves by
    // more than 8 leaves e^-8 of what was summed, so few factors ever matter, and they are formed in 64 bits.
    float base = -kInf;
    double sum = 0.0;    // (tiles are summed in 32 bits, and their sums in 64: chains of eight, however long the row)
    float bar = -kLargest;
    int n = 0;           // entries of the wave's list
    auto load = [&](int t0, BeamTile<LOADS>& f) {
        if (t0 + kTile <= end) {  // a whole tile: requests without conditions
#pragma unroll
            for (int u = 0; u < LOADS; ++u) f.raw[u] = gload16_any(logits + (size_t)(t0 + (u * kWave + lane) * E) * kSize);
            return;
        }
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int i = t0 + (u * kWave + lane) * E;
            if (i + E <= end) f.raw[u] = gload16_any(logits + (size_t)i * kSize);
        }
    };
    float x[LOADS][E], most[LOADS];  // a tile's values, and the largest of each sixteen bytes
    auto values = [&](int t0, const BeamTile<LOADS>& f) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) unpack<DTYPE>(f.raw[u], x[u]);
        if (t0 + kTile > end) {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const int i = t0 + (u * kWave + lane) * E;
                if (i + E <= end) continue;
#pragma unroll
                for (int e = 0; e < E; ++e) x[u][e] = i + e < end ? logit<DTYPE>(logits, i + e) : -kInf;
            }
        }
        // A NaN makes the tile's sum one, +infinity too: then the values are formed again, without them.
        float grown, next, all;
        for (bool again = false;; again = true) {
            grown = top;
            all = 0.0f;
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                most[u] = x[u][0];
#pragma unroll
                for (int e = 1; e < E; ++e) most[u] = fmaxf(most[u], x[u][e]);
                grown = fmaxf(grown, most[u]);
            }
            next = grown > base + 8.0f ? grown : base;
            const float from = next == -kInf ? 0.0f : next;
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                float part = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) part += __builtin_amdgcn_exp2f((x[u][e] - from) * kLog2e);
                all += part;
            }
            if (again || __ballot(all != all) == 0) break;
#pragma unroll
            for (int u = 0; u < LOADS; ++u)
#pragma unroll
                for (int e = 0; e < E; ++e) x[u][e] = fminf(fmaxf(x[u][e], -kInf), kLargest);  // (a NaN becomes -infinity)
        }
        if (__ballot(next != base && sum != 0.0)) sum *= exp_of((double)base - (double)next);
        sum += (double)all;
        base = next;
        top = grown;
    };
    // waves of this slice that have a tile, and how many values each vouches for
    const int active = min(kBeamWaves, (end - begin + kTile - 1) / kTile), quota = (a.take + active - 1) / active;
    auto share = [&](uint32_t q) {
        if (lane == 0) reinterpret_cast<volatile uint32_t*>(shares)[wave] = q;
    };
    auto shared_bar = [&]() {
        const volatile uint64_t* p = shares;
        const uint64_t a = p[0], b = p[1];
        // (a NaN where a wave has too few values: the comparison with it leaves the bar)
        return value_of(min(min((uint32_t)a, (uint32_t)(a >> 32)), min((uint32_t)b, (uint32_t)(b >> 32))));
    };
    // Entries from which on the list is looked at.  us, 512 rows of 131072, one threshold from the first tile on / this / no candidates at all: in fp32,
    // 64 taken 63 / 59 / 47, 8 taken 60 / 51 / 48, in bf16, 16 taken 43 / 38 / 29.
    int limit = min(kWave, max(16, 2 * quota));
    auto push = [&](int t0) {
        float best = most[0];
#pragma unroll
        for (int u = 1; u < LOADS; ++u) best = fmaxf(best, most[u]);
        if (__ballot(best >= bar) == 0) return;
        uint32_t late = 0;  // loads whose values the list has no room for
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            if (__ballot(most[u] >= bar) == 0) continue;
            uint64_t mask[E];
            int more = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) mask[e] = __ballot(x[u][e] >= bar), more += __popcll(mask[e]);
            if (n + more > kList) {
                late |= 1u << u;
                continue;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (mask[e] == 0) continue;
                if (x[u][e] >= bar) list[n + __popcll(mask[e] & ((1ull << lane) - 1))] = entry_of(x[u][e] + 0.0f, t0 + (u * kWave + lane) * E + e);
                n += __popcll(mask[e]);
            }
        }
        const bool cut = late != 0;
        while (late) {  // these come from memory once more, one value per lane at a time
            const int u = __builtin_ctz(late);
            late &= late - 1;
#pragma unroll 1
            for (int e = 0; e < E; ++e) {
                const int i = t0 + (u * kWave + lane) * E + e;
                const float y = i < end ? fminf(fmaxf(logit<DTYPE>(logits, i), -kInf), kLargest) + 0.0f : -kInf;
                if (n + kWave > kList) {  // (of this tile lower tokens may still come with the same value)
                    bar = fmaxf(bar, value_of(cut_parts<DTYPE, kListParts>(list, n, a.take, token_bits)));
                    n = a.take;
                }
                const uint64_t mask = __ballot(y >= bar);
                if (y >= bar) list[n + __popcll(mask & ((1ull << lane) - 1))] = entry_of(y, i);
                n += __popcll(mask);
            }
        }
        if (n <= limit && !cut) return;
        // a better q, and what does not reach the threshold any more leaves the list
        auto shorten = [&](auto parts_) {
            constexpr int N = decltype(parts_)::value;
            uint32_t hi[N];
            uint64_t v[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[j] = j * kWave + lane < n ? list[j * kWave + lane] : 0;
                hi[j] = (uint32_t)(v[j] >> 32);
            }
            if constexpr (N == 1) share(wave_kth_few(hi[0], quota));
            else share(wave_kth(hi, quota, 12));
            const float reach = shared_bar();
            bar = fmaxf(bar, reach);
            n = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const bool keep = v[j] != 0 && !(value_of(hi[j]) < reach);  // (not `bar`, which may lie above entries that stay)
                const uint64_t mask = __ballot(keep);
                if (keep) list[n + __popcll(mask & ((1ull << lane) - 1))] = v[j];
                n += __popcll(mask);
            }
        };
        if (n <= kWave) shorten(std::integral_constant<int, 1>());
        else shorten(std::integral_constant<int, kListParts>());
        if (n > 2 * kWave || (cut && n >= a.take)) {  // (the waves' threshold may have left fewer)
            // tokens of later tiles lose to those of the list that have the same value
            bar = fmaxf(bar, value_of(cut_parts<DTYPE, kListParts>(list, n, a.take, token_bits) + 1));
            n = a.take;
        }
        limit = max(limit, n + quota + 8);
    };
    const int stride = kBeamWaves * kTile;
    BeamTile<LOADS> now, next;
    int t0 = begin + wave * kTile;
    load(t0, now);
#pragma unroll 1
    for (bool first = true; first || t0 < end; t0 += stride, first = false) {
        const bool there = t0 < end;  // (a wave without a tile only meets the others)
        load(t0 + stride, next);
        if (there) values(t0, now);
        if (first) {
            uint32_t q = 0xffffffffu;
            if (there) {
                float best = most[0];
#pragma unroll
                for (int u = 1; u < LOADS; ++u) best = fmaxf(best, most[u]);
                q = wave_kth_few(order_of(best + 0.0f), quota);
            }
            share(q);
            __syncthreads();
            bar = fmaxf(bar, shared_bar());
        }
        if (there) push(t0);
        now = next;
    }
    // ---- the four waves meet
    if (n > kWave) {
        cut_parts<DTYPE, kListParts>(list, n, a.take, token_bits);
        n = a.take;
    }
    const float all = quad_max(row16_allreduce_max(top));
    sum = wave_sum64(sum * exp_of((double)base - (double)all));
    if (lane == 0) {
        wave_sums[wave] = BeamSum{all, score, sum};
        kept[wave] = n;
    }
    __syncthreads();
    if (wave != 0) return;
    float m = -kInf;
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < kBeamWaves; ++k) m = fmaxf(m, wave_sums[k].top);
#pragma unroll
    for (int k = 0; k < kBeamWaves; ++k) s += wave_sums[k].sum * (double)__builtin_amdgcn_exp2f((wave_sums[k].top - (m == -kInf ? 0.0f : m)) * kLog2e);
    for (int k = 1; k < kBeamWaves; ++k) {
        if (lane < kept[k]) list[n + lane] = lists[k][lane];
        n += kept[k];
    }
    __builtin_amdgcn_wave_barrier();
    if (n > kWave) {
        cut_parts<DTYPE, kListParts>(list, n, a.take, token_bits);
        n = a.take;
    } else if (n > a.take) {
        sort_few(list, n);
        n = a.take;
    }
    __builtin_amdgcn_wave_barrier();
    if (lane == 0) a.sums[blockIdx.x] = BeamSum{m, score, s};
    if (lane < a.take) a.best[(size_t)blockIdx.x * a.take + lane] = lane < n ? list[lane] : 0;
}

// over eight neighbouring lanes: those one and two away, and the mirrored ones of the other half
__device__ __forceinline__ uint32_t eight_max(uint32_t x) {
    x = max(x, (uint32_t)dpp_movi<0xB1>((int)x));
    x = max(x, (uint32_t)dpp_movi<0x4E>((int)x));
    return max(x, (uint32_t)dpp_movi<0x141>((int)x));
}
__device__ __forceinline__ int eight_sum(int x) {
    x += dpp_movi<0xB1>(x);
    x += dpp_movi<0x4E>(x);
    return x + dpp_movi<0x141>(x);
}

// log s to 1e-10 (the library's logarithm is four times the code): s = 2^e f with f between sqrt(1/2) and sqrt(2), and
// log f = 2 artanh(z) = 2 (z + z^3 / 3 + z^5 / 5 + ...) with z = (f - 1) / (f + 1), at most 0.172
__device__ __forceinline__ double log_of(double s) {
    double f = __builtin_amdgcn_frexp_mant(s);  // 1/2 .. 1
    int e = __builtin_amdgcn_frexp_exp(s);
    if (f < 0.70710678) f *= 2.0, --e;
    const double z = (f - 1.0) / (f + 1.0), y = z * z;
    const double p = 1.0 + y * (1.0 / 3 + y * (1.0 / 5 + y * (1.0 / 7 + y * (1.0 / 9 + y * (1.0 / 11)))));
    return (double)e * 0.69314718055994531 + 2.0 * z * p;
}

// A workgroup per group.
constexpr int kGroupThreads = 1024, kSubs = kGroupThreads / 16;
constexpr int kGroupList = 1024;  // candidates that reach the group's threshold and are ordered at a time
__device__ __forceinline__ bool before(double c, int row, uint64_t e, double c2, int row2, uint64_t e2) {
    return c > c2 || (c == c2 && (row < row2 || (row == row2 && e > e2)));
}
__global__ __launch_bounds__(kGroupThreads) void beam_groups_kernel(BeamArgs a) {
    constexpr float kInf = __builtin_inff();
    __shared__ double log_sum[kBeamRows];
    __shared__ float row_top[kBeamRows], row_score[kBeamRows];
    __shared__ uint8_t row_kind[kBeamRows];  // 0: offers nothing, 1: tokens, 2: its end
    __shared__ __attribute__((aligned(16))) uint32_t set_top[kGroupThreads / 8];
    __shared__ double list_c[kGroupList];
    __shared__ __attribute__((aligned(16))) uint32_t list_key[kGroupList];  // of c in binary32; 0 behind the last
    __shared__ uint64_t list_e[kGroupList];
    __shared__ int16_t list_row[kGroupList];
    __shared__ uint32_t bar_order;
    __shared__ int listed;
    const int tid = threadIdx.x, group = blockIdx.x;
    // Sixteen lanes take a row, or several times sixteen where rows are fewer: `parts` of them each
    const int sub = tid >> 4, sixteenth = tid & 15;
    const int per_row = a.slices * a.take, parts = a.beams < kSubs ? kSubs / a.beams : 1;
    auto first_entry = [&](int r, int part) {
        const int k = part * 16 + sixteenth;
        return k < per_row ? a.best[(size_t)(group * a.beams + r) * per_row + k] : 0;
    };
    auto entries = [&](int r, int part, uint64_t first, auto&& f) {
        const uint64_t* best = a.best + (size_t)(group * a.beams + r) * per_row;
        if (first) f(first);
#pragma unroll 2
        for (int k = (part + parts) * 16 + sixteenth; k < per_row; k += parts * 16) {
            const uint64_t e = best[k];
            if (e) f(e);
        }
    };
    auto value = [&](int r, uint64_t e) {
        return (double)row_score[r] + (((double)value_of((uint32_t)(e >> 32)) - (double)row_top[r]) - log_sum[r]);
    };
    // m and log s of the rows, and a threshold that at least `take` candidates reach: the take-th largest of the maxima of 128 sets of
    // eight threads, in binary32 rounded down
    float most = -kInf;
    auto look = [&](double c) {
        const float f = (float)c;
        most = fmaxf(most, (double)f > c ? value_of(order_of(f) - 1) : f);
    };
    for (int w = sub; w < a.beams * parts; w += kSubs) {
        const int r = w / parts, row = group * a.beams + r;
        const BeamSum* sums = a.sums + (size_t)row * a.slices;
        const bool has = sixteenth < a.slices;
        // (asked for before it is known whether the row has any)
        const BeamSum mine = sums[has ? sixteenth : 0];
        const uint64_t first = first_entry(r, w - r * parts);
        const float score = mine.score;
        const bool alive = score > -kInf, ended = mine.sum == kBeamDone;
        float m = -kInf;
        double s = 0.0;
        if (alive && !ended) {
            if (has) m = mine.top;
            for (int k = sixteenth + 16; k < a.slices; k += 16) m = fmaxf(m, sums[k].top);
            m = row16_allreduce_max(m);
            const float base = m == -kInf ? 0.0f : m;
            if (has) s = mine.sum * (double)__builtin_amdgcn_exp2f((mine.top - base) * 1.4426950408889634f);
            for (int k = sixteenth + 16; k < a.slices; k += 16) s += sums[k].sum * (double)__builtin_amdgcn_exp2f((sums[k].top - base) * 1.4426950408889634f);
            s = dpp_add64<0x121>(dpp_add64<0x122>(dpp_add64<0x124>(dpp_add64<0x128>(s))));
        }
        // (every lane and part of a row writes the same)
        row_top[r] = m;
        log_sum[r] = s > 0.0 ? log_of(s) : 0.0;
        row_score[r] = score;
        const int kind = !alive ? 0 : ended ? 2 : m > -kInf ? 1 : 0;
        row_kind[r] = kind;
        if (kind == 2 && w == r * parts && sixteenth == 0) look((double)score);
        if (kind == 1) entries(r, w - r * parts, first, [&](uint64_t e) { look(value(r, e)); });
    }
    // the threshold of every thread's `most`
    auto threshold = [&]() {
        const uint32_t v = eight_max(order_of(most));
        if ((tid & 7) == 0) set_top[tid >> 3] = v;
        __syncthreads();
        // eight neighbouring threads place their set among the 128: sixteen comparisons each
        const int set = tid >> 3, k0 = (tid & 7) * 16;
        int rank = 0;
#pragma unroll
        for (int k = 0; k < 16; k += 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(&set_top[k0 + k]);
            rank += (x.x > v || (x.x == v && k0 + k < set)) + (x.y > v || (x.y == v && k0 + k + 1 < set));
            rank += (x.z > v || (x.z == v && k0 + k + 2 < set)) + (x.w > v || (x.w == v && k0 + k + 3 < set));
        }
        if (eight_sum(rank) == a.take - 1) bar_order = v;  // (one set's eight threads)
        __syncthreads();
        return (double)value_of(bar_order);
    };
    auto each = [&](auto&& f) {  // f(row, c, entry)
        for (int w = sub; w < a.beams * parts; w += kSubs) {
            const int r = w / parts, kind = row_kind[r];
            if (kind == 2 && w == r * parts && sixteenth == 0) f(r, (double)row_score[r], entry_of(0.0f, a.eos));
            if (kind == 1) entries(r, w - r * parts, first_entry(r, w - r * parts), [&](uint64_t e) { f(r, value(r, e), e); });
        }
    };
    list_key[tid] = 0;
    if (tid == 0) listed = 0;
    double bar = threshold();
#pragma unroll 1
    for (;;) {
        each([&](int r, double c, uint64_t e) {
            if (!(c >= bar)) return;
            const int at = atomicAdd(&listed, 1);
            if (at < kGroupList) list_c[at] = c, list_e[at] = e, list_row[at] = (int16_t)r, list_key[at] = order_of((float)c);
        });
        __syncthreads();
        if (listed <= kGroupThreads / 4) break;
        // Where few rows have all of the best, few sets do: a threshold of what was listed, which lies in no order, is higher.  (One beam of 32
        // that counts, 64 taken: 26 us without it.)
        most = -kInf;
        if (tid < listed) look(list_c[tid]);
        const double higher = threshold();
        if (!(higher > bar)) break;  // ties: what was listed stays
        bar = higher;
        list_key[tid] = 0;
        if (tid == 0) listed = 0;
        __syncthreads();
    }
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
        // eight neighbouring threads count what comes before a candidate, by c in binary32 and, where others have the same, in full
        for (int i = tid >> 3; i < n; i += kGroupThreads / 8) {
            const uint32_t key = list_key[i];
            int rank = 0, same = 0;
            for (int k = 4 * (tid & 7); k < n; k += 32) {
                const uint4 x = *reinterpret_cast<const uint4*>(&list_key[k]);
                rank += (x.x > key) + (x.y > key) + (x.z > key) + (x.w > key);
                same += (x.x == key) + (x.y == key) + (x.z == key) + (x.w == key);
            }
            const double c = list_c[i];
            const uint64_t e = list_e[i];
            const int row = list_row[i];
            if (same > (int)(((i >> 2) & 7) == (tid & 7)))  // others than itself
                for (int k0 = 4 * (tid & 7); k0 < n; k0 += 32)
                    for (int k = k0; k < k0 + 4; ++k) rank += list_key[k] == key && before(list_c[k], list_row[k], list_e[k], c, row, e);
            rank = eight_sum(rank);
            if ((tid & 7) == 0 && rank < a.take) write(rank, c, row, e);
        }
    } else {
        // more than the list holds: every candidate that reaches the threshold against all others
        each([&](int r, double c, uint64_t e) {
            if (!(c >= bar)) return;
            int rank = 0;
            for (int r2 = 0; r2 < a.beams && rank < a.take; ++r2) {
                if (row_kind[r2] == 0) continue;
                if (row_kind[r2] == 2) {
                    rank += before((double)row_score[r2], r2, entry_of(0.0f, a.eos), c, r, e);
                    continue;
                }
                const uint64_t* best = a.best + (size_t)(group * a.beams + r2) * per_row;
                for (int k = 0; k < per_row && rank < a.take; ++k) {
                    const uint64_t e2 = best[k];
                    rank += e2 != 0 && before(value(r2, e2), r2, e2, c, r, e);
                }
            }
            if (rank < a.take) write(rank, c, r, e);
        });
    }
    if (tid >= listed && tid < a.take) {
        a.score_out[out + tid] = -kInf;
        a.parent[out + tid] = -1;
        a.token[out + tid] = -1;
        if (a.done_out) a.done_out[out + tid] = 0;
    }
}

}  // namespace

// Tiles of one load per lane where these are few: a wave's way is shorter then; else of four.  us, one / four, 16-bit logits: 4 rows of
// 32000 4.6 / 5.8, 64 rows 5.8 / 7.2, 120 rows of 50257 12.2 / 8.9, 128 rows of 65536 12.0 / 8.7.
// A slice is a multiple of what a workgroup's four waves take at a time, as large as leaves every compute unit four workgroups.
BeamCut beam_cut(int rows, int vocab, int dtype) {
    const int one = kBeamWaves * kWave * (dtype == 2 ? 4 : 8);
    const int64_t groups = 4ll * num_cus();
    BeamCut c;
    c.loads = (int64_t)rows * ((vocab + one - 1) / one) <= groups + groups / 2 ? 1 : 4;
    const int step = c.loads * one, steps = (vocab + step - 1) / step;
    const int64_t want = c.loads == 1 ? 2 * groups : groups;
    int64_t slices = rows > 0 ? (want + rows - 1) / rows : 1;
    if (slices > steps) slices = steps;
    const int per = (int)((steps + slices - 1) / slices);
    c.slices = (steps + per - 1) / per;
    c.slice = per * step;
    return c;
}

namespace {
template <int DTYPE>
void rows_instance(const BeamArgs& a, int loads, hipStream_t st) {
    const dim3 grid(a.groups * a.beams * a.slices), wg(kBeamThreads);
    if (loads == 4) beam_rows_kernel<DTYPE, 4><<<grid, wg, 0, st>>>(a);
    else beam_rows_kernel<DTYPE, 1><<<grid, wg, 0, st>>>(a);
}
}  // namespace

hipError_t launch_beam_rows(const BeamArgs& a, int dtype, int loads, hipStream_t st) {
    if (dtype == 0) rows_instance<0>(a, loads, st);
    else if (dtype == 1) rows_instance<1>(a, loads, st);
    else rows_instance<2>(a, loads, st);
    return hipGetLastError();
}
hipError_t launch_beam_groups(const BeamArgs& a, hipStream_t st) {
    beam_groups_kernel<<<dim3(a.groups), dim3(kGroupThreads), 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace floe
