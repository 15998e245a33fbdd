// Attention of a few query rows per sequence over the paged 8-bit cache (decoding, drafted tokens, short chunks).
//
// Mathematics, for the query rows r = (token, head of the group) that share a KV head:
//   t_rj = scale * log2(e) * (q_r . kcode_j) * kscale_j + log2(vscale_j)      o_r = sum_j 2^t_rj vcode_j / sum_j 2^(t_rj) / vscale_j
// i.e. the softmax with the scale of V inside the exponent: codes go to the matrix cores as they are (int8 and e4m3 are exact in
// fp16), no product with a scale is formed per element, and the largest weight that V is multiplied with is a fixed power of two
// whatever the scales are.  The exponent's base of a row is set so that its largest weight is 2^14, and set again only when a weight would
// pass 2^15 (after the first tokens it hardly ever is): fp16 holds the weights, down to 2^-38 of the largest.  Their rounding is what
// the result is off by beside its own: 2.2e-4 of it in all with fp16 outputs (2.1e-4 is the rounding of the output), 2.5e-4 when the
// base is set to 2^7, which costs 1 % less time on long prompts.  Queries in bf16 are scaled per row by a power of two into fp16's range.
//
// The sum below the line does without V's scale, and the scales of a sequence can lie 181 powers of two apart (2^-60 is an append's least
// one, a block of the largest bf16 values has 2^121): a token whose weight times scale binary32 no longer holds can have all of the
// softmax.  Who has walked over scales that lie further apart than 2^80 forms its sum once more, without them and with the base that the
// rows ended with; below that, what is lost is less than 2^-44 of a row's sum.  (A branch for it in the walk costs prompts 4 %, this 0 to
// 1, at 192 dims 3.)  Sums are kept times 2^20, which puts the largest weight of a row between 2^-88 and 2^95, and two of them meet on one
// base in two steps.
//
// S^T = K Q^T and O^T = V^T P^T, both as v_mfma_f32_16x16x32_f16: a column is a query row, so its maximum and sum live in the four
// lanes that hold the column, and the rows of S^T that a lane holds (tokens 4 g + i of two tiles) are exactly the operand of the
// second product when V is stored in that order: the weights never leave their lane.
//
// What bounds it: the bytes of the cache, and for few short sequences the way to the first of them.  A workgroup takes one chunk of
// one segment (sequence, KV head, tile of rows); its four waves take the chunk's units of 32 tokens in turn, one unit ahead in registers,
// and meet in LDS at the end.  A segment of one chunk is finished there; the others leave a partial result per chunk, which
// kv_join_kernel joins.  The card deals out the workgroups, so ragged batches and single long sequences fill it alike.
#pragma once

#include "kv_launch.h"

namespace floe {

constexpr int kRowsWaves = 4;
constexpr float kBaseBits = 14.0f, kTopBits = 15.0f;  // a row's largest weight is 2^14 when its base is set, and may grow to 2^15
constexpr float kSumBits = 20.0f, kSumUnit = 0x1p20f;  // sums of weights are kept times 2^20

// V's scale as the attention uses it: an append writes no smaller one, and 0 (of an array that was filled in another way) has no logarithm.
__device__ __forceinline__ float v_scale_of(float scale) { return scale < kKvFloor ? kKvFloor : scale; }  // (a NaN stays one)
// The least and the largest scale of V that a wave has walked over, as bits in scalar registers (they are positive; a NaN is a large one).
struct KvSpread {
    int least = 0x7f800000, most = 0;
    __device__ __forceinline__ void take(float scale) {
        const int bits = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, scale));
        least = min(least, bits);
        most = max(most, bits);
    }
    __device__ __forceinline__ bool wide() const { return most - least > 80 << 23; }
};

// Units of one sequence: `tiles` tiles of rows per KV head, `units` units of 32 tokens from token `lo` on for each.
struct KvUnits {
    KvSpan span;
    int tiles, units, lo;
};
template <int MT>
__device__ __forceinline__ KvUnits kv_units(const KvAttnArgs& a, int seq) {
    KvUnits u;
    u.span = kv_span(a.s, seq);
    if (u.span.rows > a.most_rows) u.span.rows = 0;  // the prompt kernel's
    u.tiles = (u.span.rows * a.group + 16 * MT - 1) / (16 * MT);
    u.lo = a.window > 0 ? max(0, u.span.pos0 - a.window + 1) & ~(kKvGroup - 1) : 0;
    const int end = a.causal ? max(0, u.span.pos0 + u.span.rows) : u.span.len;  // behind the last token that any row sees
    u.units = max(0, end - u.lo + kKvGroup - 1) / kKvGroup;
    return u;
}
// Chunks of a segment: a.chunk units each; the last of the a.chunks that the launch has takes whatever is left.
__device__ __forceinline__ int kv_chunks(const KvAttnArgs& a, int units) { return min(max(1, (units + a.chunk - 1) / a.chunk), a.chunks); }

// A wave's loads of V are whole lines that nobody reads again: without a place in the caches they leave it to K, whose lines two loads
// share.  us, none / V / K / both so: 64 sequences to 16000 tokens 238 220 233 228, one of 131001 53.8 49.4 49.1 47.2, 32 of 1600 to 4096
// (e4m3, with the append) 47.3 41.9 44.7 45.9, 16 heads of their own 21.6 21.5 23.2 23.9.
__device__ __forceinline__ uint4 gload16_once(const void* p) {
    const u32x4 q = __builtin_nontemporal_load((const FLOE_GLOBAL u32x4*)p);
    return make_uint4(q.x, q.y, q.z, q.w);
}

template <int D, int FMT>
struct KvFrag {  // one unit in registers
    uint4 k[2 * (D / 64)];
    uint4 v[D / 32];
    float ks, vs;
};

template <int D, int FMT, bool WITH_V = true>
__device__ __forceinline__ void load_unit(KvFrag<D, FMT>& f, const KvCache& c, int head, int page, int token_in_page, int r, int g) {
    const size_t slot = (size_t)max(page, 0) * c.heads + head;
    const size_t base = (slot * c.block + token_in_page) * D;  // the same in every lane
    const unsigned char *k = scalar_ptr(c.k + base), *v = scalar_ptr(c.v + base);
    const uint32_t k_lane = r * D + 16 * g, v_lane = r * 64 + 16 * g;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < D / 64; ++kk) f.k[t * (D / 64) + kk] = gload16(k + (k_lane + t * 16 * D + kk * 64));
    if constexpr (WITH_V) {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) f.v[dt] = gload16_once(v + (v_lane + dt * 1024));
    }
    f.ks = gloadf(c.k_scale + slot);
    f.vs = gloadf(c.v_scale + slot);
}

// A row of bf16 queries is multiplied with the power of two that gives its largest exponent 14 (2^14 <= largest < 2^15): an
// element below 2^-31 of the largest loses bits of its eight then, below 2^-38 all of them.  Zeros, infinities and NaN stay as they are.
struct PowerOfTwo {
    float up, down;
};
__device__ __forceinline__ PowerOfTwo bring_to_fp16(float largest) {
    const int e = (int)(__builtin_bit_cast(uint32_t, largest) >> 23) - 127;
    const int up = (e == 128 || largest == 0.0f) ? 0 : min(14 - e, 126);
    return PowerOfTwo{__builtin_bit_cast(float, (uint32_t)(127 + up) << 23), __builtin_bit_cast(float, (uint32_t)(127 - up) << 23)};
}
__device__ __forceinline__ uint32_t largest_bf16(uint4 q) {  // of the absolute values, as bits
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max(top, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
    return top;
}
__device__ __forceinline__ h16x8 bf16_to_h8(uint4 q, float f) {
    float x[8];
    unpack8<true>(q, x);
    h16x8 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const h16x2 p = __builtin_convertvector(f32x2{x[2 * j] * f, x[2 * j + 1] * f}, h16x2);
        r[2 * j] = p.x;
        r[2 * j + 1] = p.y;
    }
    return r;
}

// One query row's eight halves of a reduction step, in the order in which the codes of K arrive; rows without a query are zero.
template <int D, int MT>
struct KvQueries {
    h16x8 q[MT][D / 32];
    float unscale[MT];  // what the row was divided by
};
template <int D, int MT>
__device__ __forceinline__ void load_queries(KvQueries<D, MT>& Q, const KvAttnArgs& a, const KvSpan& span, int head, int row0, int r, int g) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int rr = row0 + 16 * m + r;
        const bool there = rr < span.rows * a.group;
        const int token = there ? rr / a.group : 0, h = there ? rr - token * a.group : 0;
        const uint16_t* p = a.q + (span.row0 + token) * a.q_stride + (size_t)(head * a.group + h) * D + 16 * g;
        Q.unscale[m] = 1.0f;
        uint4 raw[D / 32];
#pragma unroll
        for (int s = 0; s < D / 32; ++s) raw[s] = there ? gload16(p + (s >> 1) * 64 + (s & 1) * 8) : make_uint4(0, 0, 0, 0);
        if (!a.bf16) {
#pragma unroll
            for (int s = 0; s < D / 32; ++s) Q.q[m][s] = __builtin_bit_cast(h16x8, raw[s]);
            continue;
        }
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) top = max(top, largest_bf16(raw[s]));
        const PowerOfTwo f = bring_to_fp16(quad_max(bf16_to_f32(top)));
        Q.unscale[m] = f.down;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) Q.q[m][s] = bf16_to_h8(raw[s], f.up);
    }
}

// Running state of 16 MT query rows: column r of the tiles, tokens 4 g + i in lane (r, g).
template <int D, int MT>
struct KvState {
    f32x4 o[MT][D / 16];  // O^T: tile dt, parity e: dims 32 dt + 8 g + 2 i + e in o[2 dt + e][i]
    float top[MT], sum[MT];
    KvSpread spread;
};

// S^T of a unit: row r of tile m in s[m][t][i], token 16 t + 4 g + i
template <int D, int FMT, int MT>
__device__ __forceinline__ void unit_scores(f32x4 (&s)[MT][2], const KvQueries<D, MT>& Q, const KvFrag<D, FMT>& f) {
#pragma unroll
    for (int m = 0; m < MT; ++m) s[m][0] = s[m][1] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < D / 64; ++kk) {
            const uint4 c = f.k[t * (D / 64) + kk];
            const h16x8 k0 = codes_to_h8<FMT>(c.x, c.y), k1 = codes_to_h8<FMT>(c.z, c.w);
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                s[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, Q.q[m][2 * kk], s[m][t], 0, 0, 0);
                s[m][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, Q.q[m][2 * kk + 1], s[m][t], 0, 0, 0);
            }
        }
}
__device__ __forceinline__ void mask_unit(float (&x)[8], int token0, int first_key, int last_key, int g) {
    const bool none = last_key < first_key;
    const int lo = (none ? token0 + 2 * kKvGroup : first_key) - (token0 + 4 * g);  // keys from here on, up to `more` behind, are seen
    const uint32_t more = none ? 0 : last_key - first_key;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (uint32_t)(16 * (j >> 2) + (j & 3) - lo) > more ? -__builtin_inff() : x[j];
}

template <int D, int FMT, int MT>
__device__ __forceinline__ void take_unit(KvState<D, MT>& st, const KvQueries<D, MT>& Q, const KvFrag<D, FMT>& f, const KvAttnArgs& a,
                                          bool mask, int token0, int len, const int* first_key, const int* last_key, int g) {
    f32x4 s[MT][2];
    unit_scores<D, FMT, MT>(s, Q, f);
    const float vs = v_scale_of(f.vs), lv = __builtin_amdgcn_logf(vs), rv = __builtin_amdgcn_rcpf(vs) * kSumUnit;
    st.spread.take(vs);
    h16x8 p[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const float c = a.scale_log2 * Q.unscale[m] * f.ks;
        float x[8], mx = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf(s[m][j >> 2][j & 3], c, lv);
        if (mask) mask_unit(x, token0, first_key[m], last_key[m], g);
#pragma unroll
        for (int j = 0; j < 8; ++j) mx = fmaxf(mx, x[j]);
        mx = quad_max(mx);
        const bool move = mx > st.top[m] + kTopBits;
        if (__ballot(move)) {
            const float top = move ? mx - kBaseBits : st.top[m], shrink = move ? __builtin_amdgcn_exp2f(st.top[m] - top) : 1.0f;
            st.sum[m] *= shrink;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) st.o[m][d] *= shrink;
            st.top[m] = top;
        }
        const float base = st.top[m] == -__builtin_inff() ? 0.0f : st.top[m];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = __builtin_amdgcn_exp2f(x[j] - base);
            sum += x[j];
        }
        // (a block whose scale is NaN counts only where something of it is seen)
        const float add = sum * rv;
        st.sum[m] += sum != 0.0f ? add : 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const h16x2 p2 = __builtin_convertvector(f32x2{x[2 * j], x[2 * j + 1]}, h16x2);
            p[m][2 * j] = p2.x;
            p[m][2 * j + 1] = p2.y;
        }
    }
    // codes behind the last token are whatever the page held before (e4m3 has NaN): they become zeros
    uint4 vc[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) vc[dt] = f.v[dt];
    if (mask) {
        const int n0 = min(max(len - token0 - 4 * g, 0), 4), n1 = min(max(len - token0 - 16 - 4 * g, 0), 4);
        const uint32_t keep0 = n0 == 4 ? ~0u : (1u << (8 * n0)) - 1u, keep1 = n1 == 4 ? ~0u : (1u << (8 * n1)) - 1u;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) vc[dt].x &= keep0, vc[dt].y &= keep1, vc[dt].z &= keep0, vc[dt].w &= keep1;
    }
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
        const uint4 c = vc[dt];
        const h16x8 v0 = codes_to_h8<FMT>(c.x, c.y), v1 = codes_to_h8<FMT>(c.z, c.w);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            st.o[m][2 * dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[m], st.o[m][2 * dt], 0, 0, 0);
            st.o[m][2 * dt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[m], st.o[m][2 * dt + 1], 0, 0, 0);
        }
    }
}

// A unit's weights, summed without V's scale
template <int D, int FMT, int MT>
__device__ __forceinline__ void sum_unit(KvState<D, MT>& st, const KvQueries<D, MT>& Q, const KvFrag<D, FMT>& f, const KvAttnArgs& a, int token0,
                                         const int* first_key, const int* last_key, int g) {
    f32x4 s[MT][2];
    unit_scores<D, FMT, MT>(s, Q, f);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const float c = a.scale_log2 * Q.unscale[m] * f.ks;
        const float off = kSumBits - (st.top[m] == -__builtin_inff() ? 0.0f : st.top[m]) + (f.vs == f.vs ? 0.0f : f.vs);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf(s[m][j >> 2][j & 3], c, off);
        mask_unit(x, token0, first_key[m], last_key[m], g);
#pragma unroll
        for (int j = 0; j < 8; ++j) st.sum[m] += __builtin_amdgcn_exp2f(x[j]);
    }
}

__device__ __forceinline__ float weight_of(float top, float all) { return top == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(top - all); }

// The same in two steps, for sums of weights: what a sum is multiplied with can be less than binary32 holds.
__device__ __forceinline__ float half_weight_of(float top, float all) { return top == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(0.5f * (top - all)); }

// four dims of a finished row
__device__ __forceinline__ void write_row4(const KvAttnArgs& a, int D, size_t row, int head, int d, f32x4 o, float top, float sum) {
    const float f = sum == 0.0f ? 0.0f : kSumUnit / sum;
    uint2 w;
    if (a.bf16) w = make_uint2(pack16<true>(o[0] * f, o[1] * f), pack16<true>(o[2] * f, o[3] * f));
    else w = make_uint2(pack16<false>(o[0] * f, o[1] * f), pack16<false>(o[2] * f, o[3] * f));
    *reinterpret_cast<uint2*>(a.out + (row * a.q_heads + head) * D + d) = w;
    if (a.lse && d == 0)
        a.lse[row * a.q_heads + head] = sum == 0.0f ? -__builtin_inff() : (top + __builtin_amdgcn_logf(sum * (1.0f / kSumUnit))) * 0.6931471805599453f;
}

template <int D, int FMT, int MT>
__global__ __launch_bounds__(64 * kRowsWaves, kv_rows_waves_per_simd(D, MT)) void kv_rows_kernel(KvAttnArgs a) {
    constexpr int NW = kRowsWaves, kStride = D + 4;
    __shared__ float slab[NW][16][kStride];
    __shared__ float ml[NW][16 * MT][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
    // (quotients are formed in vector registers: what all lanes hold alike goes back to scalar ones)
    const int segments = a.c.heads * a.tiles, seq = __builtin_amdgcn_readfirstlane(blockIdx.x / segments);
    const int seg = blockIdx.x - seq * segments, chunk = blockIdx.y;
    const int head = __builtin_amdgcn_readfirstlane(seg / a.tiles), tile = seg - head * a.tiles, row0 = tile * 16 * MT;
    const KvUnits w = kv_units<MT>(a, seq);
    const int n_chunks = __builtin_amdgcn_readfirstlane(kv_chunks(a, w.units));
    if (tile >= w.tiles || chunk >= n_chunks) return;
    const int j0 = chunk * a.chunk, j1 = chunk + 1 < n_chunks ? j0 + a.chunk : w.units;
    KvState<D, MT> st;
    int first_key[MT], last_key[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        st.top[m] = -__builtin_inff();
        st.sum[m] = 0.0f;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) st.o[m][d] = f32x4{0, 0, 0, 0};
        const int token = min((row0 + 16 * m + r) / a.group, w.span.rows - 1), pos = w.span.pos0 + token;
        first_key[m] = a.window > 0 ? max(0, pos - a.window + 1) : 0;
        last_key[m] = a.causal ? pos : w.span.len - 1;
    }
    // units between these need no mask
    const int pos0 = w.span.pos0 + row0 / a.group;
    const int pos1 = w.span.pos0 + min((row0 + 16 * MT - 1) / a.group, w.span.rows - 1);
    const int clear_lo = __builtin_amdgcn_readfirstlane(a.window > 0 ? pos1 - a.window + 1 : 0);
    const int clear_hi = __builtin_amdgcn_readfirstlane(a.causal ? pos0 + 1 : w.span.len);  // first token that some row does not see
    const int end = __builtin_amdgcn_readfirstlane(a.causal ? pos1 + 1 : w.span.len);       // behind the last token that any row sees
    const int unit0 = w.lo / kKvGroup, log_upb = a.c.block == 32 ? 0 : a.c.block == 64 ? 1 : 2;  // units per block: 1, 2 or 4
    int pages = -1;
    auto fetch_pages = [&](int j) {  // pages of this wave's next 64 units
        const int mine = j + NW * lane;
        pages = mine < j1 ? kv_page(a.s, a.c, seq, (unit0 + mine) >> log_upb) : -1;
    };
    auto page_of = [&](int it) { return __builtin_amdgcn_readlane(pages, it & 63); };
    const int n = (j1 - j0 - wave + NW - 1) / NW;  // units of this wave (may be none)
    KvFrag<D, FMT> f0, f1;  // a unit at work and the next on its way
    int p0 = -1, p1 = -1;
    // (without a condition: a wait behind a request that may not have been made is a wait for everything; the last unit comes again)
    auto request = [&](int next, KvFrag<D, FMT>& f, int& page) {
        const int it = min(next, n - 1), j = j0 + wave + NW * it;
        if ((it & 63) == 0 && it == next) fetch_pages(j);
        page = w.lo + j * kKvGroup >= end ? -1 : page_of(it);
        load_unit<D, FMT>(f, a.c, head, page, ((unit0 + j) & ((1 << log_upb) - 1)) * kKvGroup, r, g);
    };
    if (n > 0) {
        request(0, f0, p0);
        KvQueries<D, MT> Q;
        load_queries<D, MT>(Q, a, w.span, head, row0, r, g);
        auto step = [&](int it, const KvFrag<D, FMT>& f, int page, KvFrag<D, FMT>& fill, int& fill_page) {
            request(it + 1, fill, fill_page);
            if (it >= n || page < 0) return;
            const int token0 = w.lo + (j0 + wave + NW * it) * kKvGroup;
            take_unit<D, FMT, MT>(st, Q, f, a, token0 < clear_lo || token0 + kKvGroup > clear_hi, token0, w.span.len, first_key, last_key, g);
        };
        for (int it = 0; it < n; it += 2) {
            step(it, f0, p0, f1, p1);
            step(it + 1, f1, p1, f0, p0);
        }
        if (st.spread.wide()) {
#pragma unroll
            for (int m = 0; m < MT; ++m) st.sum[m] = 0.0f;
            for (int it = 0; it < n; ++it) {
                const int j = j0 + wave + NW * it;
                if ((it & 63) == 0) fetch_pages(j);
                const int page = w.lo + j * kKvGroup >= end ? -1 : page_of(it);
                if (page < 0) continue;
                load_unit<D, FMT, false>(f0, a.c, head, page, ((unit0 + j) & ((1 << log_upb) - 1)) * kKvGroup, r, g);
                sum_unit<D, FMT, MT>(st, Q, f0, a, w.lo + j * kKvGroup, first_key, last_key, g);
            }
        }
    }
    // ---- the four waves meet
    const bool whole = n_chunks == 1;
    const size_t part0 = ((size_t)blockIdx.x * a.chunks + chunk) * a.part_rows;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        st.sum[m] = quad_sum(st.sum[m]);
        if (g == 0) {
            ml[wave][16 * m + r][0] = st.top[m];
            ml[wave][16 * m + r][1] = st.sum[m];
        }
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        float all_top = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < NW; ++i) all_top = fmaxf(all_top, ml[i][16 * m + r][0]);
        const float f0 = weight_of(st.top[m], all_top);
        if (m) __syncthreads();  // the slab of the tile before is read
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            float* at = &slab[wave][r][32 * dt + 8 * g];
            *reinterpret_cast<f32x4*>(at) = f32x4{st.o[m][2 * dt][0], st.o[m][2 * dt + 1][0], st.o[m][2 * dt][1], st.o[m][2 * dt + 1][1]} * f0;
            *reinterpret_cast<f32x4*>(at + 4) = f32x4{st.o[m][2 * dt][2], st.o[m][2 * dt + 1][2], st.o[m][2 * dt][3], st.o[m][2 * dt + 1][3]} * f0;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const int id = tid + 64 * NW * i, row = id / (D / 4), d = (id - row * (D / 4)) * 4, rr = row0 + 16 * m + row;
            if (rr >= w.span.rows * a.group) continue;
            float top = -__builtin_inff(), l = 0.0f;
            f32x4 o = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < NW; ++k) top = fmaxf(top, ml[k][16 * m + row][0]);
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                const float w = half_weight_of(ml[k][16 * m + row][0], top);
                l += ml[k][16 * m + row][1] * w * w;
                o += *reinterpret_cast<const f32x4*>(&slab[k][row][d]);
            }
            if (whole) {
                const int token = rr / a.group;
                write_row4(a, D, w.span.row0 + token, head * a.group + rr - token * a.group, d, o, top, l);
            } else {
                const size_t at = part0 + 16 * m + row;
                *reinterpret_cast<f32x4*>(a.parts.o + at * D + d) = o;
                if (d == 0) *reinterpret_cast<f32x2*>(a.parts.ml + 2 * at) = f32x2{top, l};
            }
        }
    }
}

// Joins the `n` partial results of one query row of one head, which lie at `first`, first + step, ...: a workgroup of 256 threads, of
// which 256 / (D / 4) partial results are read side by side.
template <int D>
__device__ __forceinline__ void join_row(const KvAttnArgs& a, const KvParts& parts, size_t first, int step, int n, size_t row, int head) {
    constexpr int kLanes = D / 4, kSide = 256 / kLanes;
    __shared__ f32x4 so[kSide][kLanes];
    __shared__ float sm[kSide], sl[kSide];
    const int tid = threadIdx.x, lane = tid % kLanes, side = tid / kLanes;
    float top = -__builtin_inff(), l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    if (side < kSide) {
        for (int c = side; c < n; c += kSide) {
            const size_t at = first + (size_t)c * step;
            const float t = parts.ml[2 * at], s = parts.ml[2 * at + 1];
            const f32x4 x = *reinterpret_cast<const f32x4*>(parts.o + at * D + 4 * lane);
            const float m = fmaxf(top, t), h0 = half_weight_of(top, m), h1 = half_weight_of(t, m);
            o = o * (h0 * h0) + x * (h1 * h1);
            l = l * h0 * h0 + s * h1 * h1;
            top = m;
        }
        so[side][lane] = o;
        if (lane == 0) sm[side] = top, sl[side] = l;
    }
    __syncthreads();
    if (side != 0) return;
#pragma unroll
    for (int i = 1; i < kSide; ++i) {
        const float m = fmaxf(top, sm[i]), h0 = half_weight_of(top, m), h1 = half_weight_of(sm[i], m);
        o = o * (h0 * h0) + so[i][lane] * (h1 * h1);
        l = l * h0 * h0 + sl[i] * h1 * h1;
        top = m;
    }
    write_row4(a, D, row, head, 4 * lane, o, top, l);
}
// A workgroup per query row and head, of the segments that have several chunks.
template <int D, int MT>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttnArgs a) {
    const int seq = blockIdx.y, head_q = blockIdx.x % a.q_heads, token = blockIdx.x / a.q_heads;
    const KvUnits w = kv_units<MT>(a, seq);
    if (token >= w.span.rows) return;
    const int n_chunks = kv_chunks(a, w.units);
    if (n_chunks == 1) return;  // finished where it was formed
    const int head = head_q / a.group, rr = token * a.group + head_q - head * a.group, tile = rr / (16 * MT);
    const size_t segment = ((size_t)seq * a.c.heads + head) * a.tiles + tile;
    join_row<D>(a, a.parts, segment * a.chunks * a.part_rows + rr - tile * 16 * MT, a.part_rows, n_chunks, w.span.row0 + token, head_q);
}

}  // namespace floe
