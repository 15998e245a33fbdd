// Bookkeeping of the paged cache's pages: reordering of tables, handing out with copy on write, giving back, packing, copying.
//
// A pool is nothing but a count per page of the table entries that name it; a page is free where its count is not positive.  Counts go up
// and down by integer atomics, whose order does not show, and pages are handed out from the lowest on to requests in the order of
// (sequence, block): the same state and the same call give the same tables.
#include "kv_pages.h"

namespace floe {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ bool is_page(const KvPool& p, int e) { return (unsigned)e < (unsigned)p.n_pages; }
__device__ __forceinline__ int length_of(const int32_t* len, int seq) { return min(max(len[seq], 0), kKvMaxLen); }
__device__ __forceinline__ void add_ref(const KvPool& p, int page, int by) {
    __hip_atomic_fetch_add(p.refs + page, by, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---- reorder: workgroups of the first n_seqs rows change the counts of what a source names, the others write the tables of the children.
// A source with one child changes no count: only those that ended and those with several go to their pages.
constexpr int kReorderEntries = 2 * kThreads;  // of a row, per workgroup
__global__ __launch_bounds__(kThreads) void kv_reorder_kernel(KvPool p, KvTable t, const int32_t* len, const int32_t* parent, KvTable out, int32_t* len_out) {
    const int row = blockIdx.x, tid = threadIdx.x, first = blockIdx.y * kReorderEntries;
    if (row < t.n_seqs) {
        __shared__ int total;
        if (tid == 0) total = 0;
        __syncthreads();
        int children = 0;
        for (int i = tid; i < out.n_seqs; i += kThreads) children += parent[i] == row;
        if (children) atomicAdd(&total, children);
        __syncthreads();
        const int change = total - 1;
        if (change == 0) return;
        for (int b = first + tid; b < min(first + kReorderEntries, t.max_blocks); b += kThreads) {
            const int e = t.at[(size_t)row * t.max_blocks + b];
            if (is_page(p, e)) add_ref(p, e, change);
        }
        return;
    }
    const int child = row - t.n_seqs, from = parent[child];
    const bool there = (unsigned)from < (unsigned)t.n_seqs;
    for (int b = first + tid; b < min(first + kReorderEntries, out.max_blocks); b += kThreads)
        out.at[(size_t)child * out.max_blocks + b] = there ? t.at[(size_t)from * t.max_blocks + b] : -1;
    if (first == 0 && tid == 0) len_out[child] = there ? len[from] : 0;
}

// ---- trim: a thread per table entry
__global__ __launch_bounds__(kThreads) void kv_trim_kernel(KvPool p, KvTable t, const int32_t* len, int sinks, int window) {
    const int seq = blockIdx.x, b = blockIdx.y * kThreads + threadIdx.x;
    if (b >= t.max_blocks) return;
    int32_t* at = t.at + (size_t)seq * t.max_blocks + b;
    const int e = *at, end = length_of(len, seq);
    const uint32_t first = (uint32_t)b * p.block;  // (up to 2^31)
    const int last = (int)min(first + p.block, (uint32_t)end);  // behind the block's last token
    const bool keep = first < (uint32_t)end && (window == 0 || last > end - window + 1 || first < (uint32_t)sinks);
    if (keep) return;
    if (is_page(p, e)) add_ref(p, e, -1);
    if (e != -1) *at = -1;
}

// ---- reserve: one workgroup
constexpr int kReserveThreads = 1024, kReserveWaves = kReserveThreads / kWave;
// sum over the threads before this one, and over all
__device__ __forceinline__ int workgroup_scan(int x, int* waves, int& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, up_to = wave_inclusive_scan(x);
    __syncthreads();  // (`waves` may still be read from the call before)
    if (lane == 63) waves[wave] = up_to;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int i = 0; i < kReserveWaves; ++i) {
        const int n = waves[i];
        before += i < wave ? n : 0;
        all += n;
    }
    return before + up_to - x;
}
__device__ __forceinline__ int load_agent(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void meet_in_memory() {  // what the workgroup wrote before is what its loads and atomics find behind it
    __threadfence();
    __syncthreads();
    __threadfence();
}

__global__ __launch_bounds__(kReserveThreads) void kv_reserve_kernel(KvPool p, KvTable t, const int32_t* len, const int32_t* cu, int32_t* pairs,
                                                                     int32_t* missing, KvReserveScratch w) {
    __shared__ int waves[kReserveWaves], ends[kReserveThreads], blocks[kReserveThreads];
    const int tid = threadIdx.x;
    // Every block that the call's rows touch, in order: f(sequence, block, slot) by threads that take 1024 neighbouring ones at a time
    // (f is called by all threads together; slot < 0: none).  Returns how many blocks lie behind the table.
    auto each_block = [&](auto&& f) {
        int outside = 0;
        for (int s0 = 0; s0 < t.n_seqs; s0 += kReserveThreads) {
            const int s = s0 + tid;
            int n = 0, first = 0;
            if (s < t.n_seqs) {
                const int L = length_of(len, s), rows = min(max(cu[s + 1] - cu[s], 0), kKvMaxLen);
                if (rows > 0) {
                    first = L / p.block;
                    const int behind = (int)(((uint32_t)L + rows - 1) / p.block) + 1;
                    n = max(0, min(behind, t.max_blocks) - first);
                    outside = min(outside + (behind - first - n), 1 << 20);  // (1024 threads' stay within 31 bits)
                }
            }
            int total;
            const int before = workgroup_scan(n, waves, total);
            __syncthreads();  // (the arrays may still be read)
            ends[tid] = before + n;
            blocks[tid] = first - before;
            __syncthreads();
            for (int slot0 = 0; slot0 < total; slot0 += kReserveThreads) {
                const int slot = slot0 + tid;
                int lo = 0;
                if (slot < total) {
                    int hi = kReserveThreads - 1;
                    while (lo < hi) {  // the first sequence whose blocks end behind the slot
                        const int mid = (lo + hi) >> 1;
                        if (ends[mid] > slot) hi = mid;
                        else lo = mid + 1;
                    }
                }
                f(s0 + lo, blocks[lo] + slot, slot < total);
            }
        }
        return outside;
    };
    auto entry = [&](int s, int b) { return t.at + (size_t)s * t.max_blocks + b; };
    // pages with more than one name
    bool any = false;
    for (int s = tid; s < t.n_seqs; s += kReserveThreads) pairs[2 * s] = pairs[2 * s + 1] = -1;
    const int mine_outside = each_block([&](int s, int b, bool there) {
        if (!there) return;
        const int e = *entry(s, b);
        if (!is_page(p, e)) return;
        if (p.refs[e] <= 1) return;
        w.first[e] = 0x7fffffff;
        w.writers[e] = 0;
        any = true;
    });
    int outside;
    workgroup_scan(mine_outside, waves, outside);
    meet_in_memory();
    if (__syncthreads_or(any)) {
        each_block([&](int s, int b, bool there) {
            if (!there) return;
            const int e = *entry(s, b);
            if (!is_page(p, e) || p.refs[e] <= 1) return;
            __hip_atomic_fetch_min(w.first + e, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_fetch_add(w.writers + e, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        });
        meet_in_memory();
    }
    // requests, in order
    int requests = 0;
    each_block([&](int s, int b, bool there) {
        int need = 0;
        if (there) {
            const int e = *entry(s, b);
            need = 1;
            if (is_page(p, e)) {
                const int names = p.refs[e];
                need = names > 1 && !(load_agent(w.first + e) == s && names <= load_agent(w.writers + e));
            }
        }
        int all;
        const int rank = requests + workgroup_scan(need, waves, all);
        if (need && rank < p.n_pages) w.list[rank] = KvRequest{s, b};
        requests += all;
    });
    meet_in_memory();
    // free pages, from the lowest on
    int served = 0;
    for (int p0 = 0; p0 < p.n_pages && served < requests; p0 += 4 * kReserveThreads) {
        const int page = p0 + 4 * tid;
        int4 names = make_int4(1, 1, 1, 1);
        if (page + 3 < p.n_pages) {
            names = *reinterpret_cast<const int4*>(p.refs + page);
        } else {
            if (page < p.n_pages) names.x = p.refs[page];
            if (page + 1 < p.n_pages) names.y = p.refs[page + 1];
            if (page + 2 < p.n_pages) names.z = p.refs[page + 2];
        }
        const int here[4] = {names.x <= 0, names.y <= 0, names.z <= 0, names.w <= 0};
        int all;
        int rank = served + workgroup_scan(here[0] + here[1] + here[2] + here[3], waves, all);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (!here[j]) continue;
            if (rank < requests) {
                const KvRequest r = w.list[rank];
                int32_t* at = entry(r.seq, r.block);
                const int old = *at, L = length_of(len, r.seq);
                if (is_page(p, old)) {
                    add_ref(p, old, -1);
                    if (r.block == L / p.block && L % p.block != 0) pairs[2 * r.seq] = old, pairs[2 * r.seq + 1] = page + j;
                }
                *at = page + j;
                p.refs[page + j] = 1;
            }
            ++rank;
        }
        served += all;
    }
    if (tid == 0) *missing = max(0, requests - served) + outside;
}

// ---- compact
// The i-th highest used page goes to the i-th lowest free one as long as that lies below it.  With U used pages in all, those are the used
// pages from U on and the free ones below U, and there are as many of the ones as of the others.
constexpr int kPerThread = kCompactChunk / kThreads;
__device__ __forceinline__ int workgroup_sum(int x, int* waves) {
    const int all = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = all;
    __syncthreads();
    return waves[0] + waves[1] + waves[2] + waves[3];
}
__global__ __launch_bounds__(kThreads) void kv_compact_count_kernel(KvPool p, int32_t* pairs, int n_pairs, KvCompactScratch w) {
    __shared__ int waves[kThreads / kWave];
    const int tid = threadIdx.x, first = blockIdx.x * kCompactChunk;
    int n = 0;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
        const int page = first + i * kThreads + tid;
        n += page < p.n_pages && p.refs[page] > 0;
    }
    n = workgroup_sum(n, waves);
    if (tid == 0) w.count[blockIdx.x] = n;
    for (int i = blockIdx.x * kThreads + tid; i < n_pairs; i += gridDim.x * kThreads) pairs[2 * i] = pairs[2 * i + 1] = -1;
}
__global__ __launch_bounds__(kThreads) void kv_compact_choose_kernel(KvPool p, int n_pairs, KvCompactScratch w) {
    __shared__ int waves[kThreads / kWave];
    const int tid = threadIdx.x, chunk = blockIdx.x, chunks = gridDim.x;
    int before = 0, used = 0;
    for (int i = tid; i < chunks; i += kThreads) {
        const int n = w.count[i];
        before += i < chunk ? n : 0;
        used += n;
    }
    before = workgroup_sum(before, waves);
    used = workgroup_sum(used, waves);
    // used pages below `used`
    int below = 0;
    const int last = used / kCompactChunk;
    for (int i = tid; i < last; i += kThreads) below += w.count[i];
    for (int page = last * kCompactChunk + tid; page < used; page += kThreads) below += p.refs[page] > 0;
    below = workgroup_sum(below, waves);
    const int moves = min(used - below, n_pairs);
    if (chunk == 0 && tid == 0) *w.moves = moves;
    for (int i = 0; i < kPerThread; ++i) {
        const int page = chunk * kCompactChunk + i * kThreads + tid;
        const bool there = page < p.n_pages, in_use = there && p.refs[page] > 0;
        const uint64_t mask = __ballot(in_use);
        const int lane = tid & 63, wave = tid >> 6;
        __syncthreads();
        if (lane == 0) waves[wave] = __popcll(mask);
        __syncthreads();
        int rank = before + __popcll(mask & ((1ull << lane) - 1));  // used pages before this one
#pragma unroll
        for (int k = 0; k < kThreads / kWave; ++k) {
            rank += k < wave ? waves[k] : 0;
            before += waves[k];
        }
        if (!there) continue;  // (barriers are met by all threads: the loop goes on)
        int code = page;
        if (in_use && page >= used) {
            const int i_high = used - 1 - rank;  // from the highest on
            if (i_high < moves) w.high[i_high] = page, code = -1 - i_high;
        } else if (!in_use && page < used) {
            const int i_low = page - rank;
            if (i_low < moves) w.low[i_low] = page;
        }
        w.code[page] = code;
    }
}
__global__ __launch_bounds__(kThreads) void kv_compact_move_kernel(KvPool p, KvTable t, int32_t* pairs, int32_t* page_map, KvCompactScratch w) {
    const size_t first = (size_t)blockIdx.x * kThreads + threadIdx.x, step = (size_t)gridDim.x * kThreads;
    const int moves = *w.moves;
    for (size_t i = first; i < (size_t)moves; i += step) {
        const int from = w.high[i], to = w.low[i];
        pairs[2 * i] = from;
        pairs[2 * i + 1] = to;
        p.refs[to] = p.refs[from];
        p.refs[from] = 0;
    }
    for (size_t i = first; i < (size_t)p.n_pages; i += step) {
        const int c = w.code[i];
        page_map[i] = c < 0 ? w.low[-1 - c] : c;
    }
    const size_t entries = (size_t)t.n_seqs * t.max_blocks;
    for (size_t i = first; i < entries; i += step) {
        const int e = t.at[i];
        if (!is_page(p, e)) continue;
        const int c = w.code[e];
        if (c < 0) t.at[i] = w.low[-1 - c];
    }
}

// ---- copy
__global__ __launch_bounds__(kThreads) void kv_copy_pages_kernel(KvCopyArgs a) {
    const int pair = blockIdx.x / a.pieces, piece = blockIdx.x - pair * a.pieces, tid = threadIdx.x;
    const int from = a.pairs[2 * pair], to = a.pairs[2 * pair + 1];
    if ((unsigned)from >= (unsigned)a.n_pages || (unsigned)to >= (unsigned)a.n_pages || from == to) return;
    const KvCopyArgs::Cache& c = a.cache[blockIdx.y];
    const int half = a.pieces >> 1;
    const bool is_v = piece >= half;
    const int at0 = (is_v ? piece - half : piece) * kCopyBytes;
    const uint8_t* src = (is_v ? c.v : c.k) + (size_t)from * a.bytes;
    uint8_t* dst = (is_v ? c.v : c.k) + (size_t)to * a.bytes;
    uint4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = at0 + (i * kThreads + tid) * 16;
        if (at < a.bytes) x[i] = gload16(src + at);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = at0 + (i * kThreads + tid) * 16;
        if (at < a.bytes) *reinterpret_cast<uint4*>(dst + at) = x[i];
    }
    if (at0 == 0) {
        float* s = is_v ? c.vs : c.ks;
        for (int h = tid; h < a.heads; h += kThreads) s[(size_t)to * a.heads + h] = s[(size_t)from * a.heads + h];
    }
}

}  // namespace

hipError_t launch_kv_reorder(const KvPool& p, const KvTable& t, const int32_t* len, const int32_t* parent, const KvTable& out, int32_t* len_out,
                             hipStream_t st) {
    const int columns = (out.max_blocks + kReorderEntries - 1) / kReorderEntries;
    const dim3 grid(t.n_seqs + out.n_seqs, columns > 0 ? columns : 1);  // (lengths follow their parents also where tables have no blocks)
    kv_reorder_kernel<<<grid, dim3(kThreads), 0, st>>>(p, t, len, parent, out, len_out);
    return hipGetLastError();
}
hipError_t launch_kv_trim(const KvPool& p, const KvTable& t, const int32_t* len, int sinks, int window, hipStream_t st) {
    kv_trim_kernel<<<dim3(t.n_seqs, (t.max_blocks + kThreads - 1) / kThreads), dim3(kThreads), 0, st>>>(p, t, len, sinks, window);
    return hipGetLastError();
}
hipError_t launch_kv_reserve(const KvPool& p, const KvTable& t, const int32_t* len, const int32_t* cu_rows, int32_t* pairs, int32_t* missing,
                             const KvReserveScratch& w, hipStream_t st) {
    kv_reserve_kernel<<<dim3(1), dim3(kReserveThreads), 0, st>>>(p, t, len, cu_rows, pairs, missing, w);
    return hipGetLastError();
}
hipError_t launch_kv_compact(const KvPool& p, const KvTable& t, int32_t* pairs, int n_pairs, int32_t* page_map, const KvCompactScratch& w,
                             hipStream_t st) {
    const int chunks = (p.n_pages + kCompactChunk - 1) / kCompactChunk;
    kv_compact_count_kernel<<<dim3(chunks), dim3(kThreads), 0, st>>>(p, pairs, n_pairs, w);
    kv_compact_choose_kernel<<<dim3(chunks), dim3(kThreads), 0, st>>>(p, n_pairs, w);
    const size_t entries = (size_t)t.n_seqs * t.max_blocks, most = entries > (size_t)p.n_pages ? entries : p.n_pages;
    const size_t groups = (most + kThreads - 1) / kThreads;
    kv_compact_move_kernel<<<dim3(groups < 4096 ? groups : 4096), dim3(kThreads), 0, st>>>(p, t, pairs, page_map, w);
    return hipGetLastError();
}
hipError_t launch_kv_copy_pages(KvCopyArgs a, int n_caches, hipStream_t st) {
    a.pieces = kv_copy_pieces(a.bytes);
    kv_copy_pages_kernel<<<dim3(a.n_pairs * a.pieces, n_caches), dim3(kThreads), 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace floe
