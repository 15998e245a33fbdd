// The pages of the paged cache (include/floe.h): launchers of the kernels that share, hand out, give back, pack and copy them (host side).
// Arguments are checked in kv_pages_api.hip before anything is enqueued.
#pragma once

#include "kv_cache.h"
#include "launch.h"

namespace floe {

struct KvPool {
    int32_t* refs;  // [n_pages]: table entries that name a page
    int n_pages, block;
};
struct KvTable {
    int32_t* at;  // [n_seqs][max_blocks]
    int n_seqs, max_blocks;
};

hipError_t launch_kv_reorder(const KvPool& p, const KvTable& t, const int32_t* len, const int32_t* parent, const KvTable& out, int32_t* len_out,
                             hipStream_t st);
hipError_t launch_kv_trim(const KvPool& p, const KvTable& t, const int32_t* len, int sinks, int window, hipStream_t st);

// A request that is to be served: the sequence and the block that need a page.
struct KvRequest {
    int32_t seq, block;
};
struct KvReserveScratch {
    int32_t *first, *writers;  // [n_pages]: of pages that several sequences name, the first one that writes, and how many do
    KvRequest* list;           // [n_pages]
};
hipError_t launch_kv_reserve(const KvPool& p, const KvTable& t, const int32_t* len, const int32_t* cu_rows, int32_t* pairs, int32_t* missing,
                             const KvReserveScratch& w, hipStream_t st);

constexpr int kFewPages = 8192, kFewEntries = 8192;  // pools and tables that one workgroup packs (eight pages per thread of 1024)
constexpr int kCompactChunk = 1024;  // pages that a workgroup of the compaction looks at
struct KvCompactScratch {
    int32_t* count;         // [chunks]: used pages
    int32_t *high, *low;    // [n_pairs]: the pages that move, from the highest on, and where they go, from the lowest on
    int32_t* code;          // [n_pages]: the page itself, or -1 - (its place in `high`)
    int32_t* moves;         // [1]
};
hipError_t launch_kv_compact(const KvPool& p, const KvTable& t, int32_t* pairs, int n_pairs, int32_t* page_map, const KvCompactScratch& w,
                             hipStream_t st);

constexpr int kCopyLoads = 4, kCopyBytes = kCopyLoads * 16 * 256;  // of a thread, sixteen bytes each, and of a workgroup
inline int kv_copy_pieces(int bytes) { return 2 * ((bytes + kCopyBytes - 1) / kCopyBytes); }  // of a page's K and V
constexpr int kCopyCaches = 64;  // of a launch
struct KvCopyArgs {
    struct Cache {
        uint8_t *k, *v;
        float *ks, *vs;
    } cache[kCopyCaches];
    const int32_t* pairs;  // [n_pairs][2]
    int n_pairs, n_pages, heads, bytes;  // bytes: of a page's codes of K (or of V)
    int pieces;            // set by the launcher
};
hipError_t launch_kv_copy_pages(KvCopyArgs a, int n_caches, hipStream_t st);

}  // namespace floe
