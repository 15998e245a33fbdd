// Attention of many query rows per sequence over the paged 8-bit cache (chunks of prompts, whole prompts).
//
// The same formula as the rows kernel (kv_rows.h), here bound by arithmetic: a workgroup of NW waves takes 32 NW query rows of one KV
// head (row = (token, head of the group)) and walks the tokens in tiles of 64.  A tile's codes are turned into fp16 once per
// workgroup, on their way into LDS, and read from there by every wave as operand of v_mfma_f32_32x32x16_f16.  S^T = K Q^T: a column is
// a query row, held by lanes l and l + 32, so the maximum needs one exchange; the rows of S^T in a lane (tokens 8 a + 4 h + b of a
// 32-token tile) are the operand of O^T = V^T P^T when the tokens of V lie in LDS in that order, so the weights stay in registers.
// Two LDS buffers: a wave converts the next tile's codes while others still multiply, one barrier per tile, and the tile after next is on
// its way from memory.
#pragma once

#include "kv_rows.h"

namespace floe {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kPromptTokens = 64;             // of a tile: two units of 32, each inside one page
template <int D, int NW>
struct PromptStage {  // a thread's share of a tile on its way: 16-byte pieces of the codes
    static constexpr int kPieces = (4 * D + 64 * NW - 1) / (64 * NW);
    uint4 k[kPieces], v[kPieces];
};

// The tokens that a tile of rows sees: `n` tiles of 64 from `start` on, cut into chunks as a.prompt_chunk says.
struct PromptRange {
    int start, n, chunks;
};
__device__ __forceinline__ PromptRange prompt_range(const KvAttnArgs& a, const KvSpan& span, int row0, int rows) {
    const int first = span.pos0 + row0 / a.group, last = span.pos0 + min((row0 + rows - 1) / a.group, span.rows - 1);
    const int end = a.causal ? last + 1 : span.len;  // behind the last token that any row sees
    PromptRange r;
    r.start = a.window > 0 ? max(0, first - a.window + 1) & ~(kPromptTokens - 1) : 0;
    r.n = max(0, (end - r.start + kPromptTokens - 1) / kPromptTokens);
    r.chunks = min(max(1, (r.n + a.prompt_chunk - 1) / a.prompt_chunk), a.prompt_chunks);
    return r;
}

// blockIdx.x: KV head, sequence, tile of rows; blockIdx.y: chunk of the tokens (one, unless the card would not be filled)
template <int D, int FMT, int NW>
__global__ __launch_bounds__(64 * NW, D >= 192 && NW == 4 ? 1 : 2) void kv_prompt_kernel(KvAttnArgs a) {
    // kSplit waves share 32 rows: each forms all of S^T and the weights, and a part of the dims of O^T (whose registers bound the waves)
    constexpr int kThreads = 64 * NW, kPieces = PromptStage<D, NW>::kPieces, kChunks = D / 8;
    constexpr int kSplit = kv_prompt_split(D), kRowWaves = NW / kSplit, kOut = D / 32 / kSplit;
    constexpr bool kEven = kPieces * kThreads == 4 * D;
    // Pieces of sixteen bytes.  Where a piece of a row lies is turned by the row's number so that sixteen neighbouring rows, which sixteen
    // lanes read at once, have it in sixteen different places of 256 bytes.
    __shared__ uint4 ldsK[2][kPromptTokens * kChunks];  // [token][chunk ^ swizzle(token)]: eight dims of a token
    __shared__ uint4 ldsV[2][D * 8];                    // [dim][chunk ^ (dim / 2) % 8]: chunk 2 s + h holds tokens 16 s + {4 h .. + 3, 8 + 4 h .. + 3}
    auto swizzle = [](int t) { return kChunks % 16 == 0 ? t & 15 : (t >> 1) & 7; };
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c32 = lane & 31, h = lane >> 5;
    const int row_wave = kSplit == 1 ? wave : wave % kRowWaves, out0 = kSplit == 1 ? 0 : wave / kRowWaves * kOut;  // this wave's rows and its first 32 dims of the output
    const int head = __builtin_amdgcn_readfirstlane(blockIdx.x % a.c.heads), rest = blockIdx.x / a.c.heads;
    const int seq = __builtin_amdgcn_readfirstlane(rest % a.s.n_seqs), tile = a.prompt_tiles - 1 - rest / a.s.n_seqs;  // the last rows of a prompt see most: they go first
    const KvSpan span = kv_span(a.s, seq);
    const int all_rows = span.rows * a.group, row0 = tile * 32 * kRowWaves;
    if (row0 >= all_rows || span.rows <= a.most_rows) return;
    const PromptRange range = prompt_range(a, span, row0, 32 * kRowWaves);
    const int chunk = blockIdx.y;
    if (chunk >= range.chunks) return;
    // (quotients are formed in vector registers: what all lanes hold alike goes back to scalar ones)
    const int start = __builtin_amdgcn_readfirstlane(range.start + chunk * a.prompt_chunk * kPromptTokens);
    const int n_tiles = __builtin_amdgcn_readfirstlane(chunk + 1 < range.chunks ? a.prompt_chunk : range.n - chunk * a.prompt_chunk);
    // ---- queries of this wave
    const int rr = row0 + 32 * row_wave + c32, token = min(rr / a.group, span.rows - 1), pos = span.pos0 + token;
    const bool there = rr < all_rows;
    const int head_q = head * a.group + (there ? rr - token * a.group : 0);
    h16x8 q[D / 16];
    float unscale = 1.0f;
    {
        const uint16_t* p = a.q + (span.row0 + token) * a.q_stride + (size_t)head_q * D + 8 * h;
        const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;  // the sign of the scale goes into the queries: larger S, larger weight
        uint4 raw[D / 16];
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            raw[s] = there ? gload16(p + 16 * s) : make_uint4(0, 0, 0, 0);
            raw[s].x ^= flip, raw[s].y ^= flip, raw[s].z ^= flip, raw[s].w ^= flip;
        }
        if (a.bf16) {
            uint32_t top = 0;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) top = max(top, largest_bf16(raw[s]));
            float x0, x1;
            swap32(bf16_to_f32(top), x0, x1);
            const PowerOfTwo f = bring_to_fp16(fmaxf(x0, x1));
            unscale = f.down;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) q[s] = bf16_to_h8(raw[s], f.up);
        } else {
#pragma unroll
            for (int s = 0; s < D / 16; ++s) q[s] = __builtin_bit_cast(h16x8, raw[s]);
        }
    }
    const float row_scale = fabsf(a.scale_log2) * unscale;
    // ---- tokens that the workgroup and this wave's rows see
    const int first_key = a.window > 0 ? max(0, pos - a.window + 1) : 0, last_key = a.causal ? pos : span.len - 1;
    const int w_first = span.pos0 + min((row0 + 32 * row_wave) / a.group, span.rows - 1);
    const int w_last = span.pos0 + min((row0 + 32 * row_wave + 31) / a.group, span.rows - 1);
    // tokens that every row of the wave sees
    const int w_clear_lo = __builtin_amdgcn_readfirstlane(a.window > 0 ? w_last - a.window + 1 : 0);
    const int w_clear_hi = __builtin_amdgcn_readfirstlane(a.causal ? w_first : span.len - 1);

    f32x16 o[kOut];
#pragma unroll
    for (int d = 0; d < kOut; ++d)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[d][j] = 0.0f;
    float top = -__builtin_inff(), sum = 0.0f;
    int page0 = -1, page1 = -1;  // of the tile at work

    const int unit0 = start / kKvGroup, log_upb = a.c.block == 32 ? 0 : a.c.block == 64 ? 1 : 2;  // units per block: 1, 2 or 4
    int pages = -1;
    auto page_of = [&](int unit) {  // page of the walk's unit-th unit of 32 tokens (0, 1, 2 ... in order), -1 where there is none
        if ((unit & 63) == 0) {
            const int t = start + (unit + lane) * kKvGroup;
            pages = t < span.len ? kv_page(a.s, a.c, seq, (t / kKvGroup) >> log_upb) : -1;
        }
        return __builtin_amdgcn_readlane(pages, unit & 63);
    };
    PromptStage<D, NW> next;
    auto request = [&](int it, const int* page) {  // codes of a tile
        const uint8_t *kp[2], *vp[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const size_t slot = (size_t)max(page[u], 0) * a.c.heads + head;
            const size_t at = (slot * a.c.block + ((unit0 + 2 * it + u) & ((1 << log_upb) - 1)) * kKvGroup) * D;
            kp[u] = scalar_ptr(a.c.k + at);
            vp[u] = scalar_ptr(a.c.v + at);
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int id = kEven ? tid + i * kThreads : min(tid + i * kThreads, 4 * D - 1);
            const int u = id / (2 * D), in = id - u * 2 * D;  // (2 D is a multiple of the wave: u is the same in a wave)
            next.k[i] = gload16((u ? kp[1] : kp[0]) + 16 * in);
            next.v[i] = gload16((u ? vp[1] : vp[0]) + 16 * in);
        }
    };
    float ks[2], vs[2];
    auto request_scales = [&](const int* page) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const size_t slot = (size_t)max(page[u], 0) * a.c.heads + head;
            const float k = gloadf(a.c.k_scale + slot), v = gloadf(a.c.v_scale + slot);
            ks[u] = page[u] < 0 ? 1.0f : k;  // (page 0 stands in for an absent one: what its scales hold is nobody's)
            vs[u] = page[u] < 0 ? 1.0f : v_scale_of(v);
        }
    };
    // Codes of V that no token of the sequence has (behind its end they are whatever the page held before, those of an absent page are
    // nobody's) become zeros: bytes to keep of the two runs of four tokens in a piece, for either unit of the tile.
    uint32_t keep[2][2] = {{~0u, ~0u}, {~0u, ~0u}};
    auto set_keep = [&](int it, const int* page) {
        const int g = tid & 3;  // (pieces of V: g is the fastest index, and a workgroup is a multiple of four threads)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int left = page[u] < 0 ? 0 : span.len - (start + it * kPromptTokens) - kKvGroup * u;
            if (left >= kKvGroup) {
                keep[u][0] = keep[u][1] = ~0u;
            } else {
                const int n0 = min(max(left - 4 * g, 0), 4), n1 = min(max(left - 16 - 4 * g, 0), 4);
                keep[u][0] = n0 == 4 ? ~0u : (1u << (8 * n0)) - 1u;
                keep[u][1] = n1 == 4 ? ~0u : (1u << (8 * n1)) - 1u;
            }
        }
    };
    auto convert = [&](int buf) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int id = tid + i * kThreads;
            if (!kEven && id >= 4 * D) break;  // (a whole wave)
            {
                const int t = id / (D / 16), c = 2 * (id - t * (D / 16));
                const uint4 w = next.k[i];
                ldsK[buf][t * kChunks + (c ^ swizzle(t))] = __builtin_bit_cast(uint4, codes_to_h8<FMT>(w.x, w.y));
                ldsK[buf][t * kChunks + ((c + 1) ^ swizzle(t))] = __builtin_bit_cast(uint4, codes_to_h8<FMT>(w.z, w.w));
            }
            {
                const int u = id / (2 * D), in = id - u * 2 * D, pair = in >> 2, g = in & 3;
                const uint32_t m0 = u ? keep[1][0] : keep[0][0], m1 = u ? keep[1][1] : keep[0][1];
                const uint4 w = make_uint4(next.v[i].x & m0, next.v[i].y & m1, next.v[i].z & m0, next.v[i].w & m1);
#pragma unroll
                for (int par = 0; par < 2; ++par) {
                    const int d = 2 * pair + par;
                    const uint4 x = __builtin_bit_cast(uint4, par ? codes_to_h8<FMT>(w.z, w.w) : codes_to_h8<FMT>(w.x, w.y));
                    uint2* row = reinterpret_cast<uint2*>(&ldsV[buf][d * 8]);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const int chunk = 2 * (2 * u + t) + (g & 1);
                        row[2 * (chunk ^ ((d >> 1) & 7)) + (g >> 1)] = t ? make_uint2(x.z, x.w) : make_uint2(x.x, x.y);
                    }
                }
            }
        }
    };
    // One pass over a tile makes 2 D / 16 + 4 kOut products per wave: S^T of its two units, then O^T of either.  Their operands come from LDS in
    // that order, kAhead of them on the way.
    constexpr int kStep = D / 16, kAhead = D == 192 ? 2 : 4;  // (D 192: four 297 us, two 285)
    // (With eight waves a wave has 256 registers, and at 192 and 256 dims 19 to 21 of them spill: 80 to 88 bytes of scratch per lane.)
    h16x8 ring[kAhead];
    auto operand = [&](int buf, int i) {
        if (i < 2 * kStep) {  // K: unit i / kStep, dims 16 (i % kStep) ..
            const int u = i / kStep, k = i % kStep;
            return __builtin_bit_cast(h16x8, ldsK[buf][(32 * u + c32) * kChunks + ((2 * k + h) ^ swizzle(c32))]);
        }
        const int j = i - 2 * kStep, k = j / kOut, d = out0 + j % kOut;  // V: tokens 16 k .., dims 32 d ..
        return __builtin_bit_cast(h16x8, ldsV[buf][(32 * d + c32) * 8 + ((2 * k + h) ^ ((c32 >> 1) & 7))]);
    };
    f32x16 s[2];
    h16x8 p[4];
    float c[2], lv[2], rv[2];
    KvSpread spread;  // of V's scales (kv_rows.h)
    // those of one unit: S^T (parts 0 and 1) or O^T (2 and 3); what is written behind a call and needs none of them goes between them
    auto products = [&](int buf, auto part_) {
        constexpr int part = decltype(part_)::value, n_here = part < 2 ? kStep : 2 * kOut;
        constexpr int first = part < 2 ? part * kStep : 2 * kStep + (part - 2) * 2 * kOut;
#pragma unroll
        for (int n = 0; n < n_here; ++n) {
            const int i = first + n;
            if constexpr (part < 2) s[part] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ring[i % kAhead], q[n], s[part], 0, 0, 0);
            else o[n % kOut] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ring[i % kAhead], p[2 * (part - 2) + n / kOut], o[n % kOut], 0, 0, 0);
            if (i + kAhead < 2 * kStep + 4 * kOut) ring[i % kAhead] = operand(buf, i + kAhead);
        }
    };
    // mask and running maximum of the tile
    auto maximum = [&](int t0, bool masked) {
        if (masked) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool poisoned = !(ks[u] == ks[u]) || !(vs[u] == vs[u]);  // a NaN scale: NaN for whoever sees a token, nothing for others
                const float poison = poisoned ? __builtin_nanf("") : 0.0f;
                const bool none = (u ? page1 : page0) < 0 || last_key < first_key;
                const int lo = (none ? t0 + 2 * kPromptTokens : first_key) - (t0 + 32 * u + 4 * h);  // keys from here on, up to `more` behind, are seen
                const uint32_t more = none ? 0 : last_key - first_key;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float x = s[u][j] + poison;
                    s[u][j] = (uint32_t)(8 * (j >> 2) + (j & 3) - lo) > more ? -__builtin_inff() : x;
                }
                if (poisoned) c[u] = 1.0f, lv[u] = 0.0f, rv[u] = 1.0f;
            }
        }
        float mx = -__builtin_inff();
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float m = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < 16; ++j) m = fmaxf(m, s[u][j]);
            mx = fmaxf(mx, __builtin_fmaf(m, c[u], lv[u]));
        }
        float x0, x1;
        swap32(mx, x0, x1);
        mx = fmaxf(x0, x1);
        const bool move = mx > top + kTopBits;
        if (__ballot(move)) {
            const float new_top = move ? mx - kBaseBits : top;
            const float f = move ? __builtin_amdgcn_exp2f(top - new_top) : 1.0f;
            sum *= f;
#pragma unroll
            for (int d = 0; d < kOut; ++d) o[d] *= f;
            top = new_top;
        }
    };
    auto weights = [&](int u) {
        const float off = lv[u] - (top == -__builtin_inff() ? 0.0f : top);
        float part = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][j], c[u], off));
            const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][j + 1], c[u], off));
            part += e0;
            part += e1;
            const h16x2 w = __builtin_convertvector(f32x2{e0, e1}, h16x2);
            p[2 * u + (j >> 3)][j & 7] = w.x;
            p[2 * u + (j >> 3)][(j & 7) + 1] = w.y;
        }
        sum += part * rv[u];
    };
    int page_next[2], page_then[2];
    if (n_tiles > 0) {
        page0 = page_of(0), page1 = page_of(1);
        const int now[2] = {page0, page1};
        request(0, now);
        request_scales(now);
        set_keep(0, now);
        convert(0);
        page_next[0] = page_of(2), page_next[1] = page_of(3);
        request(min(1, n_tiles - 1), page_next);
        set_keep(1, page_next);
    }
    for (int it = 0; it < n_tiles; ++it) {
        const int buf = it & 1, t0 = start + it * kPromptTokens;
        page_then[0] = page_of(2 * it + 4), page_then[1] = page_of(2 * it + 5);
        __syncthreads();  // this tile is in LDS, and nobody reads the one before it any more
        const bool masked = t0 < w_clear_lo || t0 + kPromptTokens - 1 > w_clear_hi || page0 < 0 || page1 < 0 || !(ks[0] * vs[0] + ks[1] * vs[1] > 0.0f);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ring[i] = operand(buf, i);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            c[u] = fmaxf(row_scale * ks[u], 0x1p-126f);  // (-infinity times it has to stay that)
            lv[u] = __builtin_amdgcn_logf(vs[u]);
            rv[u] = __builtin_amdgcn_rcpf(vs[u]) * kSumUnit;
            spread.take(vs[u]);
#pragma unroll
            for (int j = 0; j < 16; ++j) s[u][j] = 0.0f;
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);  // (a wave whose products wait goes before one that converts: 1 to 2 %)
        products(buf, std::integral_constant<int, 0>());
        products(buf, std::integral_constant<int, 1>());
        convert(buf ^ 1);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        request(min(it + 2, n_tiles - 1), page_then);
        maximum(t0, masked);
        weights(0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        products(buf, std::integral_constant<int, 2>());
        weights(1);
        __builtin_amdgcn_sched_barrier(0);
        request_scales(page_next);
        products(buf, std::integral_constant<int, 3>());
        __builtin_amdgcn_s_setprio(0);
        set_keep(it + 2, page_then);
        page0 = page_next[0], page1 = page_next[1];
        page_next[0] = page_then[0], page_next[1] = page_then[1];
    }
    if (spread.wide()) {  // the sum of weights once more, without V's scales; a wave by itself, its codes from memory
        const float off = kSumBits - (top == -__builtin_inff() ? 0.0f : top);
        sum = 0.0f;
        for (int unit = 0; unit < 2 * n_tiles; ++unit) {
            const int page = page_of(unit);
            if (page < 0) continue;
            const size_t slot = (size_t)page * a.c.heads + head;
            const uint8_t* k = a.c.k + (slot * a.c.block + ((unit0 + unit) & ((1 << log_upb) - 1)) * kKvGroup + c32) * D + 8 * h;
            f32x16 x;
#pragma unroll
            for (int j = 0; j < 16; ++j) x[j] = 0.0f;
#pragma unroll
            for (int n = 0; n < kStep; ++n) {
                const uint2 w = gload8(k + 16 * n);
                x = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes_to_h8<FMT>(w.x, w.y), q[n], x, 0, 0, 0);
            }
            const float k_scale = gloadf(a.c.k_scale + slot), v_scale = gloadf(a.c.v_scale + slot);
            const bool poisoned = !(k_scale == k_scale) || !(v_scale == v_scale);
            const float by = fmaxf(row_scale * k_scale, 0x1p-126f), from = poisoned ? __builtin_nanf("") : off;
            const bool none = last_key < first_key;
            const int lo = (none ? start + 2 * (unit + 2) * kKvGroup : first_key) - (start + unit * kKvGroup + 4 * h);
            const uint32_t more = none ? 0 : last_key - first_key;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], by, from));
                sum += (uint32_t)(8 * (j >> 2) + (j & 3) - lo) > more ? 0.0f : e;
            }
        }
    }
    swap32(sum, ks[0], ks[1]);
    sum = ks[0] + ks[1];
    if (!there) return;
    if (range.chunks == 1) {
#pragma unroll
        for (int d = 0; d < kOut; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                write_row4(a, D, span.row0 + token, head_q, 32 * (out0 + d) + 8 * j + 4 * h, f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]}, top, sum);
        return;
    }
    const size_t segment = ((size_t)seq * a.c.heads + head) * a.prompt_tiles + tile;
    const size_t at = (segment * a.prompt_chunks + chunk) * (32 * kRowWaves) + 32 * row_wave + c32;
#pragma unroll
    for (int d = 0; d < kOut; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *reinterpret_cast<f32x4*>(a.prompt_parts.o + at * D + 32 * (out0 + d) + 8 * j + 4 * h) = f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
    if (out0 == 0 && h == 0) *reinterpret_cast<f32x2*>(a.prompt_parts.ml + 2 * at) = f32x2{top, sum};
}

template <int D>
__global__ __launch_bounds__(256) void kv_prompt_join_kernel(KvAttnArgs a) {
    const int seq = blockIdx.y, head_q = blockIdx.x % a.q_heads, token = blockIdx.x / a.q_heads;
    const KvSpan span = kv_span(a.s, seq);
    if (token >= span.rows || span.rows <= a.most_rows) return;
    const int head = head_q / a.group, rr = token * a.group + head_q - head * a.group, tile = rr / a.prompt_rows;
    const PromptRange range = prompt_range(a, span, tile * a.prompt_rows, a.prompt_rows);
    if (range.chunks == 1) return;  // finished where it was formed
    const size_t segment = ((size_t)seq * a.c.heads + head) * a.prompt_tiles + tile;
    join_row<D>(a, a.prompt_parts, segment * a.prompt_chunks * a.prompt_rows + rr - tile * a.prompt_rows, a.prompt_rows, range.chunks, span.row0 + token, head_q);
}

}  // namespace floe
