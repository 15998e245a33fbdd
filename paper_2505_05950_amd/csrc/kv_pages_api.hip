// C entry points of the cache's pages (declared in include/floe.h): argument checks, workspace, launches.
#include "host_call.h"
#include "kv_pages.h"

using namespace floe;

namespace {

int check_pool(const floe_kv_pool* p) {
    if (!p || p->n_pages <= 0 || !p->refs || !aligned(p->refs, 16)) return FLOE_EINVAL;
    if (p->block != 32 && p->block != 64 && p->block != 128) return FLOE_EUNSUPPORTED;
    if (p->n_pages > (1 << 24)) return FLOE_EUNSUPPORTED;
    return FLOE_OK;
}
int check_sizes(int n_seqs, int max_blocks) {
    if (n_seqs < 0 || max_blocks < 0) return FLOE_EINVAL;
    if (n_seqs > 65535 || max_blocks > (1 << 23) || (int64_t)n_seqs * max_blocks > 0x7fffffff) return FLOE_EUNSUPPORTED;
    return FLOE_OK;
}
int check_table(const void* table, int n_seqs, int max_blocks) {
    return n_seqs == 0 || max_blocks == 0 || (table && aligned(table, 4)) ? FLOE_OK : FLOE_EINVAL;
}
bool apart(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return na == 0 || nb == 0 || x + na <= y || y + nb <= x;
}
KvPool dev_pool(const floe_kv_pool* p) { return KvPool{p->refs, p->n_pages, p->block}; }

struct ReserveWs {
    size_t writers, list, total;
};
ReserveWs reserve_ws(const floe_kv_pool* p) {
    ReserveWs w;
    w.writers = align_up((size_t)p->n_pages * 4);
    w.list = 2 * w.writers;
    w.total = w.list + align_up((size_t)p->n_pages * sizeof(KvRequest));
    return w;
}
constexpr int kMaxPairs = 1 << 30;  // of a compaction, whose kernels number the halves of pairs in 32 bits
struct CompactWs {
    size_t high, low, code, moves, total;
};
CompactWs compact_ws(const floe_kv_pool* p, int n_pairs) {
    const size_t most = n_pairs < p->n_pages ? n_pairs : p->n_pages;
    CompactWs w;
    w.high = align_up((size_t)(p->n_pages + kCompactChunk - 1) / kCompactChunk * 4);
    w.low = w.high + align_up(most * 4);
    w.code = w.low + align_up(most * 4);
    w.moves = w.code + align_up((size_t)p->n_pages * 4);
    w.total = w.moves + kAlign;
    return w;
}

}  // namespace

extern "C" {

int floe_kv_reorder(const floe_kv_pool* p, const int32_t* table, const int32_t* len, int n_seqs, int max_blocks, const int32_t* parent,
                    int32_t* table_out, int32_t* len_out, int n_out, void* stream) {
    int rc = check_pool(p);
    if (rc) return rc;
    if ((rc = check_sizes(n_seqs, max_blocks)) || (rc = check_sizes(n_out, max_blocks))) return rc;
    if ((rc = check_table(table, n_seqs, max_blocks)) || (rc = check_table(table_out, n_out, max_blocks))) return rc;
    if ((n_seqs && (!len || !aligned(len, 4))) || (n_out && (!parent || !len_out || !aligned(parent, 4) || !aligned(len_out, 4)))) return FLOE_EINVAL;
    const size_t in = (size_t)n_seqs * max_blocks * 4, out = (size_t)n_out * max_blocks * 4, len_in = (size_t)n_seqs * 4, each_out = (size_t)n_out * 4;
    if (!apart(table_out, out, table, in) || !apart(table_out, out, len, len_in) || !apart(table_out, out, parent, each_out) ||
        !apart(len_out, each_out, table, in) || !apart(len_out, each_out, len, len_in) || !apart(len_out, each_out, parent, each_out) ||
        !apart(table_out, out, len_out, each_out))
        return FLOE_EINVAL;
    if (n_seqs + n_out == 0) return FLOE_OK;
    hipStream_t st = (hipStream_t)stream;
    const KvTable from{const_cast<int32_t*>(table), n_seqs, max_blocks}, to{table_out, n_out, max_blocks};
    FLOE_LAUNCH(FLOE_KERNEL_KV_REORDER, st, launch_kv_reorder(dev_pool(p), from, len, parent, to, len_out, st));
    return FLOE_OK;
}

int floe_kv_trim(const floe_kv_pool* p, int32_t* table, const int32_t* len, int n_seqs, int max_blocks, int sinks, int window, void* stream) {
    int rc = check_pool(p);
    if (rc) return rc;
    if ((rc = check_sizes(n_seqs, max_blocks))) return rc;
    if (sinks < 0 || window < 0) return FLOE_EINVAL;
    if (sinks > kKvMaxLen || window > kKvMaxLen) return FLOE_EUNSUPPORTED;
    if (n_seqs == 0 || max_blocks == 0) return FLOE_OK;
    if (check_table(table, n_seqs, max_blocks) || !len || !aligned(len, 4)) return FLOE_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    FLOE_LAUNCH(FLOE_KERNEL_KV_TRIM, st, launch_kv_trim(dev_pool(p), KvTable{table, n_seqs, max_blocks}, len, sinks, window, st));
    return FLOE_OK;
}

size_t floe_kv_reserve_workspace_bytes(const floe_kv_pool* p) { return check_pool(p) == FLOE_OK ? reserve_ws(p).total : 0; }

int floe_kv_reserve(const floe_kv_pool* p, int32_t* table, const int32_t* len, const int32_t* cu_rows, int n_seqs, int max_blocks, int32_t* pairs,
                    int32_t* missing, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_pool(p);
    if (rc) return rc;
    if ((rc = check_sizes(n_seqs, max_blocks))) return rc;
    if (!missing || !aligned(missing, 4) || !workspace || !aligned(workspace, kAlign)) return FLOE_EINVAL;
    if (check_table(table, n_seqs, max_blocks)) return FLOE_EINVAL;
    if (n_seqs && (!len || !cu_rows || !pairs || !aligned(len, 4) || !aligned(cu_rows, 4) || !aligned(pairs, 4))) return FLOE_EINVAL;
    const ReserveWs w = reserve_ws(p);
    if (workspace_bytes < w.total) return FLOE_EWORKSPACE;
    char* base = static_cast<char*>(workspace);
    const KvReserveScratch scratch{reinterpret_cast<int32_t*>(base), reinterpret_cast<int32_t*>(base + w.writers), reinterpret_cast<KvRequest*>(base + w.list)};
    hipStream_t st = (hipStream_t)stream;
    FLOE_LAUNCH(FLOE_KERNEL_KV_RESERVE, st,
                launch_kv_reserve(dev_pool(p), KvTable{table, n_seqs, max_blocks}, len, cu_rows, pairs, missing, scratch, st));
    return FLOE_OK;
}

size_t floe_kv_compact_workspace_bytes(const floe_kv_pool* p, int n_pairs) {
    return check_pool(p) == FLOE_OK && n_pairs >= 0 && n_pairs <= kMaxPairs ? compact_ws(p, n_pairs).total : 0;
}

int floe_kv_compact(const floe_kv_pool* p, int32_t* table, int n_seqs, int max_blocks, int32_t* pairs, int n_pairs, int32_t* page_map, void* workspace,
                    size_t workspace_bytes, void* stream) {
    int rc = check_pool(p);
    if (rc) return rc;
    if ((rc = check_sizes(n_seqs, max_blocks))) return rc;
    if (n_pairs < 0 || (n_pairs && (!pairs || !aligned(pairs, 4))) || !page_map || !aligned(page_map, 4)) return FLOE_EINVAL;
    if (!workspace || !aligned(workspace, kAlign) || check_table(table, n_seqs, max_blocks)) return FLOE_EINVAL;
    if (n_pairs > kMaxPairs) return FLOE_EUNSUPPORTED;
    const CompactWs w = compact_ws(p, n_pairs);
    if (workspace_bytes < w.total) return FLOE_EWORKSPACE;
    char* base = static_cast<char*>(workspace);
    auto at = [&](size_t off) { return reinterpret_cast<int32_t*>(base + off); };
    const KvCompactScratch scratch{at(0), at(w.high), at(w.low), at(w.code), at(w.moves)};
    hipStream_t st = (hipStream_t)stream;
    FLOE_LAUNCH(FLOE_KERNEL_KV_COMPACT, st,
                launch_kv_compact(dev_pool(p), KvTable{table, n_seqs, max_blocks}, pairs, n_pairs, page_map, scratch, st));
    return FLOE_OK;
}

int floe_kv_copy_pages(const floe_kv_cache* caches, int n_caches, const int32_t* pairs, int n_pairs, void* stream) {
    if (n_caches < 0 || n_pairs < 0 || (n_caches && !caches)) return FLOE_EINVAL;
    for (int i = 0; i < n_caches; ++i) {
        const int rc = check_kv_cache(caches + i);
        if (rc) return rc;
        const floe_kv_cache &a = caches[0], &b = caches[i];
        if (a.n_pages != b.n_pages || a.kv_heads != b.kv_heads || a.head_dim != b.head_dim || a.block != b.block || a.format != b.format) return FLOE_ESHAPE;
    }
    if (n_caches == 0 || n_pairs == 0) return FLOE_OK;
    if (!pairs || !aligned(pairs, 4)) return FLOE_EINVAL;
    KvCopyArgs a{};
    a.pairs = pairs;
    a.n_pairs = n_pairs;
    a.n_pages = caches->n_pages;
    a.heads = caches->kv_heads;
    a.bytes = caches->kv_heads * caches->block * caches->head_dim;  // (at most 2^23)
    if ((int64_t)n_pairs * kv_copy_pieces(a.bytes) > kMaxGrid) return FLOE_EUNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    Bracket br(FLOE_KERNEL_KV_COPY, st);
    for (int i = 0; i < n_caches; i += kCopyCaches) {
        const int n = n_caches - i < kCopyCaches ? n_caches - i : kCopyCaches;
        for (int j = 0; j < n; ++j) a.cache[j] = KvCopyArgs::Cache{caches[i + j].k, caches[i + j].v, caches[i + j].k_scale, caches[i + j].v_scale};
        FLOE_HIP(launch_kv_copy_pages(a, n, st));
    }
    return FLOE_OK;
}

}  // extern "C"
