// C entry points of the paged 8-bit cache (declared in include/floe.h): argument checks, workspace, launches.
#include "host_call.h"
#include "kv_launch.h"

using namespace floe;

namespace {

int check_seqs(const floe_kv_seqs* s) {
    if (!s || s->n_seqs < 0 || s->n_rows < 0 || s->max_rows < 0 || s->max_blocks < 0) return FLOE_EINVAL;
    if (s->n_seqs > 65535 || s->n_rows > (1 << 24) || s->max_blocks > (1 << 24)) return FLOE_EUNSUPPORTED;
    return FLOE_OK;
}
bool nothing(const floe_kv_seqs* s) { return s->n_seqs == 0 || s->n_rows == 0 || s->max_rows == 0; }
int check_arrays(const floe_kv_seqs* s) {
    if (!s->cu_rows || !s->len || s->max_blocks == 0 || !s->block_table) return FLOE_EINVAL;
    return aligned(s->cu_rows, 4) && aligned(s->len, 4) && aligned(s->block_table, 4) ? FLOE_OK : FLOE_EINVAL;
}
KvCache dev_cache(const floe_kv_cache* c) {
    return KvCache{c->k, c->v, c->k_scale, c->v_scale, c->n_pages, c->kv_heads, c->head_dim, c->block};
}
KvSeqs dev_seqs(const floe_kv_seqs* s) {
    const int max_rows = s->max_rows < s->n_rows ? s->max_rows : s->n_rows;
    return KvSeqs{s->cu_rows, s->len, s->block_table, s->n_seqs, s->n_rows, max_rows, s->max_blocks};
}
int64_t block_tasks(const floe_kv_cache* c, const KvSeqs& s) {
    return (int64_t)s.n_seqs * kv_blocks_per_seq(s.max_rows, c->block) * c->kv_heads * 2;
}

int check_attention(const floe_kv_cache* c, const floe_kv_seqs* s, const floe_attention* a, int sinks) {
    int rc = check_kv_cache(c);
    if (rc) return rc;
    if ((rc = check_seqs(s))) return rc;
    if (!a || a->q_heads <= 0 || a->window < 0 || a->max_len < 0 || sinks < 0 || !__builtin_isfinite(a->scale)) return FLOE_EINVAL;
    if (a->q_heads % c->kv_heads != 0) return FLOE_ESHAPE;
    if (a->q_heads > 1024 || a->window > kKvMaxLen || sinks > kKvMaxLen) return FLOE_EUNSUPPORTED;
    // (the widest grid that has to do, in workgroups of 256 threads: the prompt kernel has two threads per query row of a KV head, at 256
    // dims four; the rows kernel has up to four workgroups)
    const KvSeqs k = dev_seqs(s);
    const int64_t rows = (int64_t)k.max_rows * (a->q_heads / c->kv_heads);
    if ((rows / (128 / kv_prompt_split(c->head_dim)) + 4) * k.n_seqs * c->kv_heads > kMaxGrid) return FLOE_EUNSUPPORTED;
    if ((int64_t)k.max_rows * a->q_heads > 0x7fffffff) return FLOE_EUNSUPPORTED;
    return FLOE_OK;
}
// Which kernels a call runs, and its workspace: [partial sums][their bases and sums of weights] of the rows kernel, and of the prompt kernel
struct AttnPlan {
    bool rows, prompt;
    int most_rows;  // sequences of up to so many rows are the rows kernel's
    int row_limit;  // at least the rows of any of those
    int mt, tiles, chunk, chunks, part_rows;
    int prompt_waves, prompt_rows, prompt_tiles, prompt_chunk, prompt_chunks;
    size_t rows_off, ml_off, prompt_ml_off, total;  // (the prompt kernel's come first)
};
// How segments (sequence, KV head, tile of rows) of up to `units` units of 32 tokens are cut into chunks: as many as give every compute
// unit one, of 8 to 128 units.  One chunk where that is nearly all of a segment, or little: a join costs about as much as 10 units.
// us, 32 / 8 heads of 128, chunks of 8, 16, 32, 64, 128 and whole segments: 1 sequence of 512 tokens 8.7 9.1 7.6 - - 7.6, 778: 8.9 10.5 10.2 -
// - 10.2, 4096: 10.0 11.3 14.5 21.2 32.7 31.4, 16000: 16.1 14.4 15.8 21.9 35.0 107, 131000: 85 69 64 57 56 870; 8 sequences of 2048: 13.9
// 13.5 15.5 20.8 18.8 18.9, 8000: 37 33 32 31 39 61; 32 of 2048: 37 35 32 31 29 29; 64 of 1000 to 16000: 286 250 239 236 236 245.
void cut_segments(AttnPlan& w, int64_t segments, int64_t units) {
    const int64_t cus = num_cus();
    int64_t chunk = ((segments * units + cus - 1) / cus + 7) & ~(int64_t)7;
    chunk = chunk < 8 ? 8 : chunk > 128 ? 128 : chunk;
    if (units <= chunk + chunk / 4 || units <= 20) chunk = units;
    const int64_t most = segments < kKvMostParts ? kKvMostParts / segments : 1;  // (bounds the workspace of many sequences)
    int64_t chunks = (units + chunk - 1) / chunk;
    if (chunks > most) chunks = most;
    w.chunk = (int)((units + chunks - 1) / chunks);
    w.chunks = (int)chunks;
}
// The prompt kernel's tiles of rows and their chunks: what costs least.  us, measured with n workgroups (8 heads of 256 rows, and 256 of
// them) over 1024 and 2048 tokens: the start and end of a workgroup, a tile of 64 tokens while it has the card to itself, and with all taken.
struct PromptCost {
    int waves;
    double start, alone, full;
    int slots;  // workgroups of a compute unit at a time
};
PromptCost prompt_cost(int dim, bool half) {
    if (dim == 64) return {4, 6.0, 1.15, 1.9, 2};
    if (dim == 128) return half ? PromptCost{4, 8.0, 1.5, 2.85, 2} : PromptCost{8, 11.0, 1.9, 2.7, 1};
    if (dim == 192) return half ? PromptCost{4, 10.0, 2.3, 2.4, 1} : PromptCost{8, 13.5, 2.9, 3.9, 1};
    return half ? PromptCost{4, 8.5, 2.35, 2.65, 1} : PromptCost{8, 8.5, 3.0, 3.8, 1};
}
// Four waves leave fewer compute units idle where rows are few, eight read the cache half as often.  us, 32 / 8 heads of 128, 8 / 4 waves:
// 6 sequences of 466 with one KV head 30.9 / 19.9, 12 of 446 with 16 / 8 heads 34.6 / 30.4, 2 x 2048 rows behind 4000 tokens 343 / 365;
// 40 / 5 heads of 192, 2224 rows with a window of 155: 93 / 115;
// 16 / 4 heads of 256, one prompt of 500 35.5 / 28.1, 6 of 1500 with a window of 700 140 / 204.
void cut_prompts(AttnPlan& w, int dim, int64_t heads, int64_t rows, int64_t tiles) {
    double best = -1;
    for (int half = 0; half < (dim == 64 ? 1 : 2); ++half) {
        const PromptCost t = prompt_cost(dim, half);
        const int64_t tile_rows = kv_prompt_rows(dim, t.waves), row_tiles = (rows + tile_rows - 1) / tile_rows, segments = heads * row_tiles;
        const int64_t cus = num_cus(), slots = cus * t.slots;
        for (int64_t c = 1; c <= 32 && c <= tiles && (c == 1 || segments * c <= 8 * slots); ++c) {
            const int64_t groups = segments * c, rounds = (groups + slots - 1) / slots;
            const double tile = groups <= (t.slots == 1 ? cus / 2 : cus) ? t.alone : t.full;
            // (a join costs its launch and the partial results' way to memory and back)
            const double cost = rounds * ((tiles + c - 1) / c * tile + t.start) + (c > 1 ? 5.0 + groups * tile_rows * dim * 8.0 / 5.0e6 : 0.0);
            if (best >= 0 && cost >= best) continue;
            best = cost;
            w.prompt_waves = t.waves;
            w.prompt_rows = (int)tile_rows;
            w.prompt_tiles = (int)row_tiles;
            w.prompt_chunk = (int)((tiles + c - 1) / c);
        }
    }
    w.prompt_chunks = (int)((tiles + w.prompt_chunk - 1) / w.prompt_chunk);
}
// The most tokens that `rows` rows of a sequence see: their windows, the first tokens, and what the steps of the walk take beside both
int64_t keys_of(const floe_attention* a, int sinks, int64_t rows) {
    const int64_t seen = a->window + rows + (sinks ? sinks + 127 : 0);
    return a->window > 0 && seen < a->max_len ? seen : a->max_len;
}
AttnPlan attn_plan(const floe_kv_cache* c, const floe_kv_seqs* s, const floe_attention* a, int sinks) {
    AttnPlan w{};
    w.total = kAlign;  // (so that a workspace is a workspace whichever kernels run)
    const KvSeqs k = dev_seqs(s);
    const int group = a->q_heads / c->kv_heads, most = kKvRowsLimit / group;
    w.rows = true;
    w.most_rows = w.row_limit = k.max_rows;
    if (k.max_rows > most) {
        // Sequences with few rows are the rows kernel's, unless there can be none (n_rows are too many for that) or the prompt kernel has
        // room for their tiles beside the others': then a launch costs more than it saves.
        const int64_t tile_rows = kv_prompt_rows(c->head_dim, prompt_cost(c->head_dim, false).waves);
        const int64_t tiles = k.n_seqs * ((k.max_rows * (int64_t)group + tile_rows - 1) / tile_rows) * c->kv_heads;
        w.prompt = true;
        w.rows = most > 0 && k.n_rows - (int64_t)(k.n_seqs - 1) * k.max_rows <= most && tiles > num_cus();
        w.most_rows = w.rows ? most : 0;
        w.row_limit = most;
    }
    if (w.prompt) {
        const int64_t keys = keys_of(a, sinks, k.max_rows);  // (a tile of rows sees less where they are many)
        cut_prompts(w, c->head_dim, (int64_t)k.n_seqs * c->kv_heads, (int64_t)k.max_rows * group, (keys + 63) / 64 + 1);
        if ((int64_t)a->q_heads * k.max_rows > kMaxGrid) w.prompt_chunks = 1;  // (more rows than a join has workgroups)
        if (w.prompt_chunks > 1) {
            const size_t parts = (size_t)k.n_seqs * c->kv_heads * w.prompt_tiles * w.prompt_chunks * w.prompt_rows;
            w.prompt_ml_off = align_up(parts * c->head_dim * 4);
            w.total = w.prompt_ml_off + align_up(parts * 8);
        }
    }
    if (!w.rows) return w;
    const int rows = w.row_limit * group;  // of a KV head
    w.mt = kv_rows_tiles_for(c->head_dim, rows);
    w.tiles = (rows + 16 * w.mt - 1) / (16 * w.mt);
    const int64_t segments = (int64_t)k.n_seqs * c->kv_heads * w.tiles;
    const int64_t keys = keys_of(a, sinks, w.row_limit);
    cut_segments(w, segments, (keys + kKvGroup - 1) / kKvGroup + 1);
    if (w.chunks > 1) {
        w.part_rows = rows < 16 * w.mt ? rows : 16 * w.mt;
        const size_t parts = (size_t)segments * w.chunks * w.part_rows;
        const size_t rows_off = w.total > kAlign ? w.total : 0;
        w.rows_off = rows_off;
        w.ml_off = rows_off + align_up(parts * c->head_dim * 4);
        w.total = w.ml_off + align_up(parts * 8);
    }
    return w;
}

}  // namespace

extern "C" {

int floe_rope_table(float* table, int n_positions, int rot_dim, double base, void* stream) {
    if (!table || !aligned(table, 16) || n_positions < 0 || rot_dim <= 0 || !(base > 0.0)) return FLOE_EINVAL;
    if (rot_dim % 16 != 0) return FLOE_ESHAPE;
    if (rot_dim > 256 || (int64_t)n_positions * (rot_dim / 2) > kMaxGrid * 256) return FLOE_EUNSUPPORTED;  // (a thread per pair)
    if (n_positions == 0) return FLOE_OK;
    FLOE_HIP(launch_rope_table(table, n_positions, rot_dim, base, (hipStream_t)stream));
    return FLOE_OK;
}

int floe_kv_append(const floe_kv_cache* c, const floe_kv_seqs* s, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                   const void* q, int64_t q_stride, int q_heads, void* q_out, const floe_rope* rope, void* stream) {
    int rc = check_kv_cache(c);
    if (rc) return rc;
    if ((rc = check_seqs(s))) return rc;
    const int64_t row = (int64_t)c->kv_heads * c->head_dim, limit = (int64_t)1 << 40;
    if (q_heads < 0 || k_stride < row || v_stride < row || k_stride % 8 || v_stride % 8) return FLOE_EINVAL;
    if (k_stride > limit || v_stride > limit || q_heads > 1024) return FLOE_EUNSUPPORTED;
    if (rope) {
        if (!rope->table || !aligned(rope->table, 16) || rope->n_positions <= 0 || rope->rot_dim <= 0 || !aligned(rope->positions, 4))
            return FLOE_EINVAL;
        if (rope->rot_dim % 16 != 0 || rope->rot_dim > c->head_dim) return FLOE_ESHAPE;
    }
    if (q) {
        if (!rope || q_heads == 0 || !q_out || !aligned(q, 16) || !aligned(q_out, 16)) return FLOE_EINVAL;
        if (q_stride < (int64_t)q_heads * c->head_dim || q_stride % 8) return FLOE_EINVAL;
        if (q_stride > limit) return FLOE_EUNSUPPORTED;
    }
    if (nothing(s)) return FLOE_OK;
    if ((rc = check_arrays(s))) return rc;
    if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return FLOE_EINVAL;
    const KvSeqs ds = dev_seqs(s);
    const int64_t q_groups = q ? ((int64_t)ds.n_rows + 3) / 4 : 0;
    if (block_tasks(c, ds) + q_groups > kMaxGrid) return FLOE_EUNSUPPORTED;
    KvAppendArgs a{};
    a.k = static_cast<const uint16_t*>(k);
    a.v = static_cast<const uint16_t*>(v);
    a.q = static_cast<const uint16_t*>(q);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_stride = q_stride;
    a.q_out = static_cast<uint16_t*>(q_out);
    a.q_heads = q_heads;
    if (rope) a.rope = KvRope{rope->table, rope->positions, rope->n_positions, rope->rot_dim, rope->interleaved != 0};
    hipStream_t st = (hipStream_t)stream;
    FLOE_LAUNCH(FLOE_KERNEL_KV_APPEND, st, launch_kv_append(dev_cache(c), ds, a, c->format, c->dtype == FLOE_BF16, st));
    return FLOE_OK;
}

int floe_kv_gather(const floe_kv_cache* c, const floe_kv_seqs* s, void* k_out, void* v_out, void* stream) {
    int rc = check_kv_cache(c);
    if (rc) return rc;
    if ((rc = check_seqs(s))) return rc;
    if (nothing(s)) return FLOE_OK;
    if ((rc = check_arrays(s))) return rc;
    if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16)) return FLOE_EINVAL;
    const KvSeqs ds = dev_seqs(s);
    if (block_tasks(c, ds) > kMaxGrid) return FLOE_EUNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    FLOE_LAUNCH(FLOE_KERNEL_KV_GATHER, st,
                launch_kv_gather(dev_cache(c), ds, static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out), c->format,
                                 c->dtype == FLOE_BF16, st));
    return FLOE_OK;
}

size_t floe_kv_attention_sinks_workspace_bytes(const floe_kv_cache* c, const floe_kv_seqs* s, const floe_attention* a, int sinks) {
    return check_attention(c, s, a, sinks) == FLOE_OK && !nothing(s) ? attn_plan(c, s, a, a->window > 0 ? sinks : 0).total : 0;
}
size_t floe_kv_attention_workspace_bytes(const floe_kv_cache* c, const floe_kv_seqs* s, const floe_attention* a) {
    return floe_kv_attention_sinks_workspace_bytes(c, s, a, 0);
}

int floe_kv_attention(const floe_kv_cache* c, const floe_kv_seqs* s, const floe_attention* a, const void* q, int64_t q_stride, void* out,
                      float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    return floe_kv_attention_sinks(c, s, a, 0, q, q_stride, out, lse, workspace, workspace_bytes, stream);
}

int floe_kv_attention_sinks(const floe_kv_cache* c, const floe_kv_seqs* s, const floe_attention* a, int sinks, const void* q, int64_t q_stride,
                            void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_attention(c, s, a, sinks);
    if (rc) return rc;
    if (q_stride < (int64_t)a->q_heads * c->head_dim || q_stride % 8) return FLOE_EINVAL;
    if (q_stride > (int64_t)1 << 40) return FLOE_EUNSUPPORTED;
    if (nothing(s)) return FLOE_OK;
    if ((rc = check_arrays(s))) return rc;
    if (!q || !out || !workspace || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(workspace, kAlign))
        return FLOE_EINVAL;
    if (a->window == 0) sinks = 0;  // (every row sees its first tokens)
    const AttnPlan w = attn_plan(c, s, a, sinks);
    if (workspace_bytes < w.total) return FLOE_EWORKSPACE;
    char* base = static_cast<char*>(workspace);
    KvAttnArgs k{};
    k.c = dev_cache(c);
    k.s = dev_seqs(s);
    k.q = static_cast<const uint16_t*>(q);
    k.q_stride = q_stride;
    k.out = static_cast<uint16_t*>(out);
    k.lse = lse;
    k.q_heads = a->q_heads;
    k.group = a->q_heads / c->kv_heads;
    k.scale_log2 = a->scale * 1.4426950408889634f;
    k.causal = a->causal != 0;
    k.window = a->window;
    k.sinks = sinks;
    k.bf16 = c->dtype == FLOE_BF16;
    k.most_rows = w.most_rows;
    k.parts = KvParts{reinterpret_cast<float*>(base + w.rows_off), reinterpret_cast<float*>(base + w.ml_off)};
    k.prompt_parts = KvParts{reinterpret_cast<float*>(base), reinterpret_cast<float*>(base + w.prompt_ml_off)};
    k.prompt_waves = w.prompt_waves;
    k.prompt_rows = w.prompt_rows;
    k.prompt_tiles = w.prompt_tiles;
    k.prompt_chunk = w.prompt_chunk;
    k.prompt_chunks = w.prompt_chunks;
    k.tiles = w.tiles;
    k.chunk = w.chunk;
    k.chunks = w.chunks;
    k.part_rows = w.part_rows;
    hipStream_t st = (hipStream_t)stream;
    const bool int8 = c->format == FLOE_KV_INT8;
    const auto prompt = sinks ? int8 ? launch_kv_prompt_sinks_int8 : launch_kv_prompt_sinks_e4m3 : int8 ? launch_kv_prompt_int8 : launch_kv_prompt_e4m3;
    const auto rows = sinks ? int8 ? launch_kv_rows_sinks_int8 : launch_kv_rows_sinks_e4m3 : int8 ? launch_kv_rows_int8 : launch_kv_rows_e4m3;
    if (w.prompt) {
        FLOE_LAUNCH(FLOE_KERNEL_KV_PROMPT, st, prompt(k, st));
        if (w.prompt_chunks > 1) FLOE_LAUNCH(FLOE_KERNEL_KV_JOIN, st, launch_kv_prompt_join(k, st));
    }
    if (w.rows) {
        FLOE_LAUNCH(FLOE_KERNEL_KV_ATTENTION, st, rows(k, w.mt, st));
        if (w.chunks > 1) FLOE_LAUNCH(FLOE_KERNEL_KV_JOIN, st, launch_kv_join(k, w.mt, w.row_limit, st));
    }
    return FLOE_OK;
}

}  // extern "C"
