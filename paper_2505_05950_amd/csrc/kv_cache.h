// The paged cache of keys and values in 8 bits, as the kernels see it (layout and arithmetic: include/floe.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "floe_dev.h"

namespace floe {

typedef _Float16 h16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kKvInt8 = 0, kKvE4m3 = 1;  // floe_kv_format
constexpr int kKvGroup = 32;             // tokens of a group of the V layout
constexpr float kKvFloor = 0x1p-60f;     // least scale of a block
constexpr int kKvMaxLen = 1 << 30;       // lengths that a kernel reads are cut to this: position arithmetic stays within 31 bits

struct KvCache {
    uint8_t* k;
    uint8_t* v;
    float* k_scale;
    float* v_scale;
    int n_pages, heads, dim, block;
};

// rows of a call: sequence s has rows cu[s] .. cu[s + 1), and a length
struct KvSeqs {
    const int32_t* cu;
    const int32_t* len;
    const int32_t* table;  // [n_seqs][max_blocks]
    int n_seqs, n_rows, max_rows, max_blocks;
};

__device__ __forceinline__ float bf16_to_f32(uint32_t low_half) { return __builtin_bit_cast(float, low_half << 16); }
__device__ __forceinline__ uint32_t f32_to_bf16(float x) {  // nearest, ties to even; a NaN stays one
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (u >> 16) | 0x40u;
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}
template <bool BF16>
__device__ __forceinline__ float from16(uint32_t low_half) {
    if constexpr (BF16) return bf16_to_f32(low_half & 0xffffu);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)low_half);
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
    if constexpr (BF16) return f32_to_bf16(a) | (f32_to_bf16(b) << 16);
    else return as_u32(__builtin_convertvector(f32x2{a, b}, h16x2));
}
template <bool BF16>
__device__ __forceinline__ void unpack8(uint4 q, float* x) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = from16<BF16>(w[j]);
        x[2 * j + 1] = from16<BF16>(w[j] >> 16);
    }
}

// Eight codes as fp16, exactly (int8 has 8 significant bits, e4m3 four, and both ranges lie inside fp16's).
// int8: code + 128 becomes the low byte of a half whose high byte is 0x64, which is 1024 + 128 + code.
template <int FMT>
__device__ __forceinline__ h16x8 codes_to_h8(uint32_t lo, uint32_t hi) {
    h16x2 p[4];
    if constexpr (FMT == kKvInt8) {
        const h16x2 off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
        lo ^= 0x80808080u;
        hi ^= 0x80808080u;
        p[0] = as_h2(__builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u)) + off;
        p[1] = as_h2(__builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u)) + off;
        p[2] = as_h2(__builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u)) + off;
        p[3] = as_h2(__builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)) + off;
    } else {
        p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
        p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
        p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
        p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    }
    return h16x8{p[0].x, p[0].y, p[1].x, p[1].y, p[2].x, p[2].y, p[3].x, p[3].y};
}
// sixteen codes as floats
template <int FMT>
__device__ __forceinline__ void codes_to_f32(uint4 c, float* x) {
    const h16x8 a = codes_to_h8<FMT>(c.x, c.y), b = codes_to_h8<FMT>(c.z, c.w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = (float)a[j];
        x[8 + j] = (float)b[j];
    }
}
// four values, already divided by the scale, as codes: nearest, ties to even, cut to the largest code
template <int FMT>
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
    if constexpr (FMT == kKvInt8) {
        const int i = (int)fminf(fmaxf(rintf(a), -127.0f), 127.0f), j = (int)fminf(fmaxf(rintf(b), -127.0f), 127.0f);
        const int k = (int)fminf(fmaxf(rintf(c), -127.0f), 127.0f), l = (int)fminf(fmaxf(rintf(d), -127.0f), 127.0f);
        return (i & 255) | ((j & 255) << 8) | ((k & 255) << 16) | ((uint32_t)l << 24);
    } else {
        a = fminf(fmaxf(a, -448.0f), 448.0f);
        b = fminf(fmaxf(b, -448.0f), 448.0f);
        c = fminf(fmaxf(c, -448.0f), 448.0f);
        d = fminf(fmaxf(d, -448.0f), 448.0f);
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
}

// Sums / maxima over the four lanes l, l ^ 16, l ^ 32, l ^ 48 by register exchange (no LDS).  The exchange swaps the second half (or the
// odd rows of 16 lanes) of its first operand with the first half (the even rows) of its second.
// (The results go through integers: a bit cast of a vector's element takes the first one whichever is named.)
__device__ __forceinline__ void swap32(float x, float& a, float& b) {
    const int u = __builtin_bit_cast(int, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t lo = r[0], hi = r[1];
    a = __builtin_bit_cast(float, lo);
    b = __builtin_bit_cast(float, hi);
}
__device__ __forceinline__ void swap16(float x, float& a, float& b) {
    const int u = __builtin_bit_cast(int, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t lo = r[0], hi = r[1];
    a = __builtin_bit_cast(float, lo);
    b = __builtin_bit_cast(float, hi);
}
__device__ __forceinline__ float quad_max(float x) {
    float a, b;
    swap32(x, a, b);
    swap16(fmaxf(a, b), a, b);
    return fmaxf(a, b);
}
__device__ __forceinline__ float quad_sum(float x) {
    float a, b;
    swap32(x, a, b);
    swap16(a + b, a, b);
    return a + b;
}

// A sequence's rows and length as a kernel may use them, whatever the arrays hold: rows inside [0, n_rows], at most max_rows of them.
// Where they are fewer than cu_rows says, they are its first ones: pos0 counts all of them.
struct KvSpan {
    int row0, rows, len;
    int pos0;  // where the first row sits if the sequence's rows are the last ones of its len tokens; at least -kKvMaxLen
};
__device__ __forceinline__ KvSpan kv_span(const KvSeqs& s, int seq) {
    const int a = max(s.cu[seq], 0), b = min(max(s.cu[seq + 1], 0), kKvMaxLen);
    KvSpan r;
    r.row0 = min(a, s.n_rows);
    r.rows = min(max(min(b, s.n_rows) - r.row0, 0), s.max_rows);
    r.len = min(max(s.len[seq], 0), kKvMaxLen);
    r.pos0 = r.len - max(b - a, 0);
    return r;
}
// page of a sequence's block, or -1 where the table names none
__device__ __forceinline__ int kv_page(const KvSeqs& s, const KvCache& c, int seq, int block) {
    if (block >= s.max_blocks) return -1;
    const int p = s.table[(size_t)seq * s.max_blocks + block];
    return (unsigned)p < (unsigned)c.n_pages ? p : -1;
}

}  // namespace floe
