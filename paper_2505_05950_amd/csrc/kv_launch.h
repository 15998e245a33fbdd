// Launchers of the kernels on the paged 8-bit cache (host side).  Arguments are checked in kv_api.hip before anything is enqueued.
#pragma once

#include "kv_cache.h"
#include "launch.h"

namespace floe {

struct KvRope {
    const float* table;        // [n_positions][rot / 2][2]
    const int32_t* positions;  // [n_rows] or nullptr: a row's place in its sequence
    int n_positions, rot, interleaved;
};

struct KvAppendArgs {
    const uint16_t *k, *v, *q;
    int64_t k_stride, v_stride, q_stride;
    uint16_t* q_out;
    int q_heads;
    KvRope rope;
    int blocks_per_seq, tasks, q_split;  // set by the launcher
};
// blocks that `rows` consecutive tokens can touch
inline int kv_blocks_per_seq(int rows, int block) { return (rows + block - 2) / block + 1; }
hipError_t launch_kv_append(const KvCache& c, const KvSeqs& s, const KvAppendArgs& a, int format, bool bf16, hipStream_t st);
hipError_t launch_kv_gather(const KvCache& c, const KvSeqs& s, uint16_t* k_out, uint16_t* v_out, int format, bool bf16, hipStream_t st);
hipError_t launch_rope_table(float* table, int n_positions, int rot, double base, hipStream_t st);

// partial results: sums of rows of `dim` values, and per row the exponent's base and the sum of the weights
struct KvParts {
    float* o;
    float* ml;
};

struct KvAttnArgs {
    KvCache c;
    KvSeqs s;  // len: tokens of each sequence, the call's own among them
    const uint16_t* q;
    int64_t q_stride;
    uint16_t* out;
    float* lse;  // [n_rows][q_heads] or nullptr
    int q_heads, group;
    float scale_log2;  // softmax scale * log2(e)
    int causal, window;
    bool bf16;
    int most_rows;  // sequences of up to so many rows are the rows kernel's, the others the prompt kernel's
    // rows kernel (kv_rows.h)
    KvParts parts;      // [n_seqs][heads][tiles][chunks][part_rows]
    int tiles;          // of 16 mt rows, per KV head
    int chunk, chunks;  // units of 32 tokens per chunk, chunks per segment
    int part_rows;      // rows of a partial result
    // prompt kernel (kv_prompt.h)
    KvParts prompt_parts;  // [n_seqs][heads][prompt_tiles][prompt_chunks][prompt_rows]
    int prompt_waves;      // of a workgroup: 4 or 8
    int prompt_rows;       // kv_prompt_rows(dim, prompt_waves)
    int prompt_tiles;      // of prompt_rows rows, per KV head
    int prompt_chunk, prompt_chunks;  // tiles of 64 tokens per chunk, chunks per tile of rows
};

constexpr int64_t kKvMostParts = 65535;  // partial results of a call
// Query rows per KV head up to which a sequence is the rows kernel's.  us, rows / prompt kernel, 32 / 8 heads of 128: 36 rows (9 tokens) of 1
// sequence of 8000 16.1 / 18.6, 8 of 8000 50 / 69, 64 of 1000 52 / 51, 1 of 1000 11.2 / 12.0; 68 rows 23.0 / 20.2, 79 / 74, 73 / 51, 12.1 / 13.4;
// 128 rows 21.4 / 23.5, 94 / 81, 100 / 57, 13.1 / 16.1.  16 / 4 heads of 256, 4 of 3000: 68 rows 29.8 / 31.1, 128 rows 40 / 34.  8 / 8 heads of 64,
// 4 of 3000: 40 rows 16.5 / 18.2, 64 rows 18.3 / 19.5.  The line is a batch's: one sequence by itself is up to 3 us behind what the rows kernel
// would take at 68 to 128 rows, where its tiles leave most of the card to none.
constexpr int kKvRowsLimit = 64;
// Tiles of sixteen rows that a workgroup of the rows kernel takes at once: as many as its registers hold beside two units of the cache
constexpr int kv_rows_most_tiles(int dim) { return dim == 64 ? 4 : dim <= 192 ? 2 : 1; }
inline int kv_rows_tiles_for(int dim, int rows) {
    const int most = kv_rows_most_tiles(dim), want = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
    return want < most ? want : most;
}
constexpr int kv_rows_waves_per_simd(int dim, int mt) { return dim * mt <= 128 ? 3 : dim * mt <= 256 && dim < 256 ? 2 : 1; }
hipError_t launch_kv_rows_int8(const KvAttnArgs& a, int mt, hipStream_t st);  // mt tiles of sixteen rows per workgroup
hipError_t launch_kv_rows_e4m3(const KvAttnArgs& a, int mt, hipStream_t st);
// prompt kernel (kv_prompt.h): how many waves share 32 query rows, rows of a workgroup
constexpr int kv_prompt_split(int dim) { return dim == 256 ? 2 : 1; }
constexpr int kv_prompt_rows(int dim, int waves) { return 32 * waves / kv_prompt_split(dim); }
hipError_t launch_kv_prompt_int8(const KvAttnArgs& a, hipStream_t st);
hipError_t launch_kv_prompt_e4m3(const KvAttnArgs& a, hipStream_t st);
hipError_t launch_kv_prompt_join(const KvAttnArgs& a, hipStream_t st);
hipError_t launch_kv_join(const KvAttnArgs& a, int mt, int rows, hipStream_t st);  // rows: at least those of any sequence it joins

}  // namespace floe
