// Appending to the paged 8-bit cache (with the rotary positions on the way) and reading tokens of it back.
//
// Mathematics: x' = x turned by the table's (cos, sin) of its position, pair by pair; need = max(amax / qmax, 2^-60) over the rows
// that this call brings to a block; scale = need for a block that it opens, else scale * 2^k with the least k that reaches need;
// code = round(x' / scale); older codes of the block: round(code * 2^-k).  Strict IEEE binary32, one rounding per operation.
#include "kv_launch.h"

namespace floe {

#pragma clang fp contract(off)

namespace {

// What a workgroup of either kernel does: the rows lo .. hi of one block (token numbers of the sequence), for one head, K or V.
struct BlockTask {
    int seq, head, page, lo, hi, first;  // first: token number of the block's first token
    bool is_v, live;
    KvSpan span;
};
__device__ __forceinline__ BlockTask block_task(const KvSeqs& s, const KvCache& c, int task, int blocks_per_seq) {
    BlockTask t;
    const int h2 = task % (2 * c.heads), rest = task / (2 * c.heads);
    t.head = h2 >> 1;
    t.is_v = h2 & 1;
    t.seq = rest / blocks_per_seq;
    t.span = kv_span(s, t.seq);
    const int block = t.span.len / c.block + rest % blocks_per_seq;
    t.first = block * c.block;
    t.lo = max(t.span.len, t.first);
    t.hi = min(t.span.len + t.span.rows, t.first + c.block);
    t.live = t.lo < t.hi;
    t.page = t.live ? kv_page(s, c, t.seq, block) : -1;
    return t;
}

// A pair unit: eight dims and the eight that they are turned with.  Units up to rot / 16 turn; the ones behind only hold 16 dims.
struct PairUnit {
    int a, b;  // first dims of the two halves
    bool turns;
};
__device__ __forceinline__ PairUnit pair_unit(int p, int rot, bool interleaved) {
    PairUnit u;
    u.turns = p < (rot >> 4);
    const bool half = u.turns && !interleaved;
    u.a = half ? 8 * p : 16 * p;
    u.b = half ? (rot >> 1) + 8 * p : 16 * p + 8;
    return u;
}
// The (cos, sin) pairs of a unit at a position: pairs of dims (a + j, b + j) in halves, (a + 2 j, a + 2 j + 1) over all sixteen when
// interleaved.  A position outside the table gives NaN, a unit that does not turn (1, 0), which leaves it as it is.
struct Turns {
    float c[8], s[8];
};
__device__ __forceinline__ Turns load_turns(const PairUnit& u, const KvRope& r, int pos) {
    Turns t;
    const bool there = (unsigned)pos < (unsigned)r.n_positions;
#pragma unroll
    for (int j = 0; j < 8; ++j) t.c[j] = u.turns && !there ? __builtin_nanf("") : 1.0f, t.s[j] = 0.0f;
    if (!u.turns || !there) return t;
    const float* at = r.table + ((size_t)pos * (r.rot >> 1) + (r.interleaved ? u.a >> 1 : u.a)) * 2;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint4 q = gload16(at + 4 * j);
        t.c[2 * j] = __builtin_bit_cast(float, q.x);
        t.s[2 * j] = __builtin_bit_cast(float, q.y);
        t.c[2 * j + 1] = __builtin_bit_cast(float, q.z);
        t.s[2 * j + 1] = __builtin_bit_cast(float, q.w);
    }
    return t;
}
// x[0..8) and x[8..16): the two halves of a unit
__device__ __forceinline__ void turn(const PairUnit& u, bool interleaved, const Turns& t, float* x) {
    if (!u.turns) return;  // (an infinity times the 0 above would not stay one)
    if (interleaved) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float p = x[2 * j], q = x[2 * j + 1];
            x[2 * j] = p * t.c[j] - q * t.s[j];
            x[2 * j + 1] = q * t.c[j] + p * t.s[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float p = x[j], q = x[8 + j];
            x[j] = p * t.c[j] - q * t.s[j];
            x[8 + j] = q * t.c[j] + p * t.s[j];
        }
    }
}

// The scale of a block behind this call, and what the older codes are divided by.  Binary32 bits are compared as integers: the largest
// of |x| over the workgroup sees infinities and NaN too, and a block that takes one has the scale NaN from then on.
struct BlockScale {
    float scale, shrink;  // shrink = 2^-k
    bool finite, grows;
};
__device__ __forceinline__ BlockScale block_scale(uint32_t amax_bits, bool opens, float old, float qmax) {
    BlockScale r;
    r.shrink = 1.0f;
    r.grows = false;
    r.finite = amax_bits < 0x7f800000u && (opens || __builtin_bit_cast(uint32_t, old) < 0x7f800000u);
    if (!r.finite) {
        r.scale = __builtin_nanf("");
        return r;
    }
    const float need = fmaxf(__builtin_bit_cast(float, amax_bits) / qmax, kKvFloor);
    r.scale = need;
    if (opens) return r;
    const uint32_t n = __builtin_bit_cast(uint32_t, need), o = __builtin_bit_cast(uint32_t, old);
    const int k = (int)(n >> 23) - (int)(o >> 23) + ((n & 0x7fffffu) > (o & 0x7fffffu) ? 1 : 0);
    r.scale = old;
    if (k > 0) {
        r.grows = true;
        r.scale = __builtin_bit_cast(float, o + ((uint32_t)k << 23));
        r.shrink = k < 127 ? __builtin_bit_cast(float, (uint32_t)(127 - k) << 23) : 0.0f;
    }
    return r;
}
// the first `n` pieces of sixteen codes of a block
template <int FMT>
__device__ __forceinline__ void recode(uint8_t* codes, int n, float shrink, int first, int step) {
    for (int id = first; id < n; id += step) {
        uint4* at = reinterpret_cast<uint4*>(codes) + id;
        float y[16];
        codes_to_f32<FMT>(*at, y);
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = codes_of<FMT>(y[4 * j] * shrink, y[4 * j + 1] * shrink, y[4 * j + 2] * shrink, y[4 * j + 3] * shrink);
        *at = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o, kWave));
    return x;
}
__device__ __forceinline__ uint32_t workgroup_max(uint32_t x, uint32_t* lds) {
    x = wave_max(x);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return max(max(lds[0], lds[1]), max(lds[2], lds[3]));
}

// The queries: a wave takes a row (or a part of its heads), its lanes the units of a few heads at a time, with the same turns.
template <bool BF16>
__device__ __forceinline__ void turn_queries(const KvCache& c, const KvSeqs& s, const KvAppendArgs& a, int id) {
    const int lane = threadIdx.x & 63, D = c.dim, row = id / a.q_split, part = id - row * a.q_split;
    if (row >= s.n_rows) return;
    int upto = 0;
    for (int i = 0; i < s.n_seqs; i += kWave) {  // sequences that begin at or before this row
        const int j = i + lane;
        upto += __popcll(__ballot(j < s.n_seqs && s.cu[min(j, s.n_seqs)] <= row));
    }
    if (upto == 0) return;
    const KvSpan span = kv_span(s, upto - 1);
    if (row - span.row0 >= span.rows) return;
    const int per_head = D >> 4, heads = kWave / per_head, first = lane / per_head;
    if (first >= heads) return;  // (D 192: 60 lanes)
    const PairUnit u = pair_unit(lane - first * per_head, a.rope.rot, a.rope.interleaved);
    const Turns t = load_turns(u, a.rope, a.rope.positions ? a.rope.positions[row] : span.len + row - span.row0);
    const uint16_t* in = a.q + row * a.q_stride;
    uint16_t* out = a.q_out + (size_t)row * a.q_heads * D;
    constexpr int kSide = 4;  // heads of a lane on their way
    const int step = a.q_split * heads;
    for (int h0 = part * heads + first; h0 < a.q_heads; h0 += kSide * step) {
        uint4 raw[kSide][2];
#pragma unroll
        for (int k = 0; k < kSide; ++k) {
            const uint16_t* at = in + min(h0 + k * step, a.q_heads - 1) * D;
            raw[k][0] = gload16(at + u.a);
            raw[k][1] = gload16(at + u.b);
        }
#pragma unroll
        for (int k = 0; k < kSide; ++k) {
            if (h0 + k * step >= a.q_heads) break;
            uint16_t* at = out + (h0 + k * step) * D;
            float x[16];
            unpack8<BF16>(raw[k][0], x);
            unpack8<BF16>(raw[k][1], x + 8);
            turn(u, a.rope.interleaved, t, x);
            *reinterpret_cast<uint4*>(at + u.a) = make_uint4(pack16<BF16>(x[0], x[1]), pack16<BF16>(x[2], x[3]), pack16<BF16>(x[4], x[5]), pack16<BF16>(x[6], x[7]));
            *reinterpret_cast<uint4*>(at + u.b) = make_uint4(pack16<BF16>(x[8], x[9]), pack16<BF16>(x[10], x[11]), pack16<BF16>(x[12], x[13]), pack16<BF16>(x[14], x[15]));
        }
    }
}

}  // namespace

// A workgroup owns one block x head of K or of V, so nobody else touches its codes and its scale: no atomics, one pass over the rows
// (they stay in registers between the maximum and the codes).  NU units of sixteen codes per thread hold what a call can bring to a
// block.  A unit of V is the sixteen bytes that lie next to each other in the cache (eight tokens x two dims): neighbouring lanes take
// the four token groups and then the next pair of dims, so a wave writes 1 KiB in one piece and reads 64 bytes of each row.  The
// workgroups behind the last task turn the queries.
template <int NU, int FMT, bool BF16>
__global__ __launch_bounds__(256) void kv_append_kernel(KvCache c, KvSeqs s, KvAppendArgs a) {
    __shared__ uint32_t lds_max[4];
    const int tid = threadIdx.x, D = c.dim;
    if ((int)blockIdx.x >= a.tasks) return turn_queries<BF16>(c, s, a, (blockIdx.x - a.tasks) * 4 + (tid >> 6));
    const BlockTask t = block_task(s, c, blockIdx.x, a.blocks_per_seq);
    if (t.page < 0) return;  // the whole workgroup
    const size_t slot = (size_t)t.page * c.heads + t.head;
    const int lo = t.lo - t.first, hi = t.hi - t.first;  // tokens of the block that this call brings
    const int row_of_0 = t.span.row0 + t.first - t.span.len;  // row of the block's token 0, were it one
    const bool opens = lo == 0;
    const float qmax = FMT == kKvInt8 ? 127.0f : 448.0f;
    float* scale_at = (t.is_v ? c.v_scale : c.k_scale) + slot;
    const float old_scale = opens ? 1.0f : *scale_at;
    uint8_t* codes = (t.is_v ? c.v : c.k) + slot * c.block * D;
    float x[NU][16];
    uint32_t amax = 0;
    if (!t.is_v) {
        const int per_row = D >> 4, new_units = (hi - lo) * per_row;
#pragma unroll
        for (int n = 0; n < NU; ++n) {
            const int id = tid + n * 256;
            if (id < new_units) {
                const int o = id / per_row, row = row_of_0 + lo + o;
                const PairUnit u = pair_unit(id - o * per_row, a.rope.rot, a.rope.interleaved);
                const int pos = a.rope.positions ? a.rope.positions[row] : t.first + lo + o;
                const uint16_t* in = a.k + row * a.k_stride + t.head * D;
                const uint4 r0 = gload16(in + u.a), r1 = gload16(in + u.b);
                const Turns turns = load_turns(u, a.rope, pos);
                unpack8<BF16>(r0, x[n]);
                unpack8<BF16>(r1, x[n] + 8);
                turn(u, a.rope.interleaved, turns, x[n]);
#pragma unroll
                for (int j = 0; j < 16; ++j) amax = max(amax, __builtin_bit_cast(uint32_t, x[n][j]) & 0x7fffffffu);
            }
        }
        const BlockScale b = block_scale(workgroup_max(amax, lds_max), opens, old_scale, qmax);
        if (tid == 0) *scale_at = b.scale;
#pragma unroll
        for (int n = 0; n < NU; ++n) {
            const int id = tid + n * 256;
            if (id < new_units) {
                const int o = id / per_row;
                const PairUnit u = pair_unit(id - o * per_row, a.rope.rot, a.rope.interleaved);
                uint32_t w[4] = {0, 0, 0, 0};
                if (b.finite) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        w[j] = codes_of<FMT>(x[n][4 * j] / b.scale, x[n][4 * j + 1] / b.scale, x[n][4 * j + 2] / b.scale, x[n][4 * j + 3] / b.scale);
                }
                uint8_t* at = codes + (size_t)(lo + o) * D;
                *reinterpret_cast<uint2*>(at + u.a) = make_uint2(w[0], w[1]);
                *reinterpret_cast<uint2*>(at + u.b) = make_uint2(w[2], w[3]);
            }
        }
        if (b.grows) recode<FMT>(codes, lo * per_row, b.shrink, tid, 256);
        return;
    }
    uint4 was[NU];
    const int unit0 = lo / kKvGroup * 2 * D, unit1 = ((hi - 1) / kKvGroup + 1) * 2 * D;  // units of the groups that get tokens
    // V: unit = ((group of 32 tokens) * D / 2 + pair of dims) * 4 + g; token 32 group + 16 tile + 4 g + i is byte 8 (dim % 2) + 4 tile + i
#pragma unroll
    for (int n = 0; n < NU; ++n) {
        const int id = unit0 + tid + n * 256;
        if (id < unit1) {
            const int g = id & 3, ap = id >> 2, group = ap / (D >> 1), pair = ap - group * (D >> 1);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int o = kKvGroup * group + 16 * (j >> 2) + 4 * g + (j & 3);
                uint32_t w = 0;
                if (o >= lo && o < hi) w = gload4(a.v + (row_of_0 + o) * a.v_stride + t.head * D + 2 * pair);
                x[n][j] = from16<BF16>(w);
                x[n][8 + j] = from16<BF16>(w >> 16);
            }
            // the codes beside new tokens, asked for before the scale is known
            const int t0 = kKvGroup * group + 4 * g;
            was[n] = make_uint4(0, 0, 0, 0);
            if (t0 < lo && t0 + 20 > lo) was[n] = gload16(codes + 16 * id);
#pragma unroll
            for (int j = 0; j < 16; ++j) amax = max(amax, __builtin_bit_cast(uint32_t, x[n][j]) & 0x7fffffffu);
        }
    }
    const BlockScale b = block_scale(workgroup_max(amax, lds_max), opens, old_scale, qmax);
    if (tid == 0) *scale_at = b.scale;
#pragma unroll
    for (int n = 0; n < NU; ++n) {
        const int id = unit0 + tid + n * 256;
        if (id >= unit1) continue;
        const int g = id & 3, group = (id >> 2) / (D >> 1);
        const int t0 = kKvGroup * group + 4 * g;  // its tokens: t0 .. t0 + 4 and t0 + 16 .. t0 + 20
        uint32_t fresh[2] = {0, 0};  // bytes of new tokens
        bool older = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int o = t0 + 16 * (j >> 2) + (j & 3);
            if (o >= lo && o < hi) fresh[j >> 2] |= 255u << (8 * (j & 3));
            older |= o < lo;
        }
        const bool brings = (fresh[0] | fresh[1]) != 0;
        if (!brings && !(older && b.grows)) continue;
        uint4* at = reinterpret_cast<uint4*>(codes) + id;
        uint32_t w[4] = {0, 0, 0, 0};
        if (older) {
            const uint4 old = t0 + 20 > lo ? was[n] : *at;
            w[0] = old.x, w[1] = old.y, w[2] = old.z, w[3] = old.w;
            if (b.grows) {  // (codes behind the block's tokens are nobody's)
                float y[16];
                codes_to_f32<FMT>(old, y);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = codes_of<FMT>(y[4 * j] * b.shrink, y[4 * j + 1] * b.shrink, y[4 * j + 2] * b.shrink, y[4 * j + 3] * b.shrink);
            }
        }
        if (brings) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t q = 0;
                if (b.finite)
                    q = codes_of<FMT>(x[n][4 * j] / b.scale, x[n][4 * j + 1] / b.scale, x[n][4 * j + 2] / b.scale, x[n][4 * j + 3] / b.scale);
                w[j] = (w[j] & ~fresh[j & 1]) | (q & fresh[j & 1]);
            }
        }
        *at = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (b.grows) recode<FMT>(codes, unit0, b.shrink, tid, 256);
}

// One token per sequence: a wave owns the block x head.  The block's maximum is a wave's, V's token is two bytes per pair of dims, and
// what lies beside them is read only where the scale grows.  What bounds it is the way from lengths to pages to scale and rows (4.4 us for
// one sequence), and the number of such ways: 98 sequences, 16 heads of 192 with the attention 29.9 us when a workgroup took each, 26.3 so.
template <int FMT, bool BF16>
__global__ __launch_bounds__(256) void kv_append_one_kernel(KvCache c, KvSeqs s, KvAppendArgs a) {
    const int lane = threadIdx.x & 63, D = c.dim, id = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (id >= a.tasks) {
        if (a.q) turn_queries<BF16>(c, s, a, id - a.tasks);
        return;
    }
    const BlockTask t = block_task(s, c, id, 1);
    if (t.page < 0) return;
    const size_t slot = (size_t)t.page * c.heads + t.head;
    const int o = t.lo - t.first, row = t.span.row0;
    const bool opens = o == 0;
    const float qmax = FMT == kKvInt8 ? 127.0f : 448.0f;
    float* scale_at = (t.is_v ? c.v_scale : c.k_scale) + slot;
    const float old_scale = opens ? 1.0f : *scale_at;
    uint8_t* codes = (t.is_v ? c.v : c.k) + slot * c.block * D;
    if (!t.is_v) {
        const int per_row = D >> 4;
        const PairUnit u = pair_unit(min(lane, per_row - 1), a.rope.rot, a.rope.interleaved);  // lanes behind the row double its last unit
        const uint16_t* in = a.k + row * a.k_stride + t.head * D;
        const uint4 r0 = gload16(in + u.a), r1 = gload16(in + u.b);
        const Turns turns = load_turns(u, a.rope, a.rope.positions ? a.rope.positions[row] : t.lo);
        float x[16];
        unpack8<BF16>(r0, x);
        unpack8<BF16>(r1, x + 8);
        turn(u, a.rope.interleaved, turns, x);
        uint32_t amax = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) amax = max(amax, __builtin_bit_cast(uint32_t, x[j]) & 0x7fffffffu);
        const BlockScale b = block_scale(wave_max(amax), opens, old_scale, qmax);
        if (lane == 0) *scale_at = b.scale;
        if (b.grows) recode<FMT>(codes, o * per_row, b.shrink, lane, kWave);
        if (lane >= per_row) return;
        uint32_t w[4] = {0, 0, 0, 0};
        if (b.finite) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = codes_of<FMT>(x[4 * j] / b.scale, x[4 * j + 1] / b.scale, x[4 * j + 2] / b.scale, x[4 * j + 3] / b.scale);
        }
        uint8_t* at = codes + (size_t)o * D;
        *reinterpret_cast<uint2*>(at + u.a) = make_uint2(w[0], w[1]);
        *reinterpret_cast<uint2*>(at + u.b) = make_uint2(w[2], w[3]);
        return;
    }
    constexpr int kPairs = 2;  // of dims per lane: head dims go up to 256
    float y[kPairs][2];
    uint32_t amax = 0;
#pragma unroll
    for (int n = 0; n < kPairs; ++n) {
        const int pair = min(lane + n * kWave, (D >> 1) - 1);  // as above
        const uint32_t w = gload4(a.v + row * a.v_stride + t.head * D + 2 * pair);
        y[n][0] = from16<BF16>(w);
        y[n][1] = from16<BF16>(w >> 16);
        amax = max(amax, max(__builtin_bit_cast(uint32_t, y[n][0]) & 0x7fffffffu, __builtin_bit_cast(uint32_t, y[n][1]) & 0x7fffffffu));
    }
    const BlockScale b = block_scale(wave_max(amax), opens, old_scale, qmax);
    if (lane == 0) *scale_at = b.scale;
    const int group = o / kKvGroup, token = o % kKvGroup;
    if (b.grows) {
        recode<FMT>(codes, (group + 1) * 2 * D, b.shrink, lane, kWave);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the new bytes come behind the pieces that other lanes wrote around them
    }
    uint8_t* at = codes + group * kKvGroup * D + ((token >> 2) & 3) * 16 + (token >> 4) * 4 + (token & 3);
#pragma unroll
    for (int n = 0; n < kPairs; ++n) {
        const int pair = lane + n * kWave;
        if (2 * pair >= D) break;
        const uint32_t w = b.finite ? codes_of<FMT>(y[n][0] / b.scale, y[n][1] / b.scale, 0.0f, 0.0f) : 0u;
        at[pair * 64] = (uint8_t)w;
        at[pair * 64 + 8] = (uint8_t)(w >> 8);
    }
}

// value = code * scale, rounded once to 16 bits; the same split and the same units as above.  Rows of absent pages are zero.
template <int FMT, bool BF16>
__global__ __launch_bounds__(256) void kv_gather_kernel(KvCache c, KvSeqs s, int blocks_per_seq, uint16_t* __restrict__ k_out,
                                                        uint16_t* __restrict__ v_out) {
    const int tid = threadIdx.x, D = c.dim;
    const BlockTask t = block_task(s, c, blockIdx.x, blocks_per_seq);
    if (!t.live) return;
    const size_t slot = (size_t)max(t.page, 0) * c.heads + t.head;
    const bool there = t.page >= 0;
    const int lo = t.lo - t.first, hi = t.hi - t.first;
    const int row_of_0 = t.span.row0 + t.first - t.span.len;
    const float scale = there ? (t.is_v ? c.v_scale : c.k_scale)[slot] : 0.0f;
    const uint4* codes = reinterpret_cast<const uint4*>((t.is_v ? c.v : c.k) + slot * c.block * D);
    const size_t out_stride = (size_t)c.heads * D;
    if (!t.is_v) {
        const int per_row = D >> 4;
        for (int id = tid; id < (hi - lo) * per_row; id += 256) {
            const int o = id / per_row, p = id - o * per_row;
            float x[16];
            codes_to_f32<FMT>(there ? gload16(codes + (lo + o) * per_row + p) : make_uint4(0, 0, 0, 0), x);
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = there ? pack16<BF16>(x[2 * j] * scale, x[2 * j + 1] * scale) : 0u;
            uint4* at = reinterpret_cast<uint4*>(k_out + (row_of_0 + lo + o) * out_stride + t.head * D + 16 * p);
            at[0] = make_uint4(w[0], w[1], w[2], w[3]);
            at[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
        return;
    }
    // a thread takes two neighbouring pairs of dims, so that sixteen lanes write a whole line of a token
    for (int id = tid; id < (c.block * D) >> 5; id += 256) {
        const int g = id & 3, ap = id >> 2, group = ap / (D >> 2), quad = ap - group * (D >> 2);
        const int t0 = kKvGroup * group + 4 * g;
        if (t0 + 20 <= lo || t0 >= hi) continue;
        const uint4* at = codes + (group * (D >> 1) + 2 * quad) * 4 + g;
        float x[16], y[16];
        codes_to_f32<FMT>(there ? gload16(at) : make_uint4(0, 0, 0, 0), x);
        codes_to_f32<FMT>(there ? gload16(at + 4) : make_uint4(0, 0, 0, 0), y);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int o = t0 + 16 * (j >> 2) + (j & 3);
            if (o >= lo && o < hi)
                *reinterpret_cast<uint2*>(v_out + (row_of_0 + o) * out_stride + t.head * D + 4 * quad) =
                    there ? make_uint2(pack16<BF16>(x[j] * scale, x[8 + j] * scale), pack16<BF16>(y[j] * scale, y[8 + j] * scale)) : make_uint2(0, 0);
        }
    }
}

// (cos, sin) of position * base^(-2 i / rot), formed in 64 bits and rounded once: in 32 a far position loses its angle
__global__ __launch_bounds__(256) void rope_table_kernel(float2* __restrict__ table, int n_positions, int rot, double base) {
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int half = rot >> 1;
    if (id >= (long long)n_positions * half) return;
    const int pos = (int)(id / half), i = (int)(id - (long long)pos * half);
    double sn, cs;
    sincos((double)pos * pow(base, -2.0 * i / rot), &sn, &cs);
    table[id] = make_float2((float)cs, (float)sn);
}

namespace {
template <int FMT, bool BF16>
hipError_t append_nu(const KvCache& c, const KvSeqs& s, const KvAppendArgs& a, hipStream_t st) {
    const int64_t turns = a.q ? (int64_t)s.n_rows * a.q_split : 0;  // waves for the queries
    if (s.max_rows == 1) {
        kv_append_one_kernel<FMT, BF16><<<dim3((unsigned)((a.tasks + turns + 3) / 4)), dim3(256), 0, st>>>(c, s, a);
        return hipGetLastError();
    }
    const int grid = a.tasks + (int)((turns + 3) / 4);
    // pieces of sixteen codes per thread: of the 32-token groups of a block that max_rows rows can touch (the registers of a whole block
    // would let a compute unit hold two workgroups)
    const int groups = (s.max_rows + 2 * kKvGroup - 2) / kKvGroup, all = c.block / kKvGroup;
    const int per_thread = ((groups < all ? groups : all) * 2 * c.dim + 255) / 256;
    if (per_thread <= 1) kv_append_kernel<1, FMT, BF16><<<dim3(grid), dim3(256), 0, st>>>(c, s, a);
    else if (per_thread <= 2) kv_append_kernel<2, FMT, BF16><<<dim3(grid), dim3(256), 0, st>>>(c, s, a);
    else if (per_thread <= 4) kv_append_kernel<4, FMT, BF16><<<dim3(grid), dim3(256), 0, st>>>(c, s, a);
    else kv_append_kernel<8, FMT, BF16><<<dim3(grid), dim3(256), 0, st>>>(c, s, a);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_kv_append(const KvCache& c, const KvSeqs& s, const KvAppendArgs& args, int format, bool bf16, hipStream_t st) {
    KvAppendArgs a = args;
    a.blocks_per_seq = kv_blocks_per_seq(s.max_rows, c.block);
    a.tasks = s.n_seqs * a.blocks_per_seq * c.heads * 2;
    // a wave per row of queries, or several where rows are few: then the way to the first of them is what there is to save
    const int passes = a.q ? (a.q_heads + kWave / (c.dim / 16) - 1) / (kWave / (c.dim / 16)) : 1;
    a.q_split = s.n_rows >= 1024 ? 1 : (1024 / s.n_rows < passes ? 1024 / s.n_rows : passes);
    if (format == kKvInt8) return bf16 ? append_nu<kKvInt8, true>(c, s, a, st) : append_nu<kKvInt8, false>(c, s, a, st);
    return bf16 ? append_nu<kKvE4m3, true>(c, s, a, st) : append_nu<kKvE4m3, false>(c, s, a, st);
}

hipError_t launch_kv_gather(const KvCache& c, const KvSeqs& s, uint16_t* k_out, uint16_t* v_out, int format, bool bf16, hipStream_t st) {
    const int bps = kv_blocks_per_seq(s.max_rows, c.block);
    const dim3 grid(s.n_seqs * bps * c.heads * 2), wg(256);
    if (format == kKvInt8) {
        if (bf16) kv_gather_kernel<kKvInt8, true><<<grid, wg, 0, st>>>(c, s, bps, k_out, v_out);
        else kv_gather_kernel<kKvInt8, false><<<grid, wg, 0, st>>>(c, s, bps, k_out, v_out);
    } else {
        if (bf16) kv_gather_kernel<kKvE4m3, true><<<grid, wg, 0, st>>>(c, s, bps, k_out, v_out);
        else kv_gather_kernel<kKvE4m3, false><<<grid, wg, 0, st>>>(c, s, bps, k_out, v_out);
    }
    return hipGetLastError();
}

hipError_t launch_rope_table(float* table, int n_positions, int rot, double base, hipStream_t st) {
    const long long n = (long long)n_positions * (rot / 2);
    rope_table_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st>>>(reinterpret_cast<float2*>(table), n_positions, rot, base);
    return hipGetLastError();
}

}  // namespace floe
