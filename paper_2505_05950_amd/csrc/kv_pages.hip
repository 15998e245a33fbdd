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

// Pages with several names among up to 1024 blocks: the first sequence of the call that writes each, and how many do (open addressing,
// half full at most).
constexpr int kNames = 2 * kReserveThreads;
struct NameTable {
    int page[kNames], first[kNames], writers[kNames];
    __device__ __forceinline__ int place(int e) {
        int at = ((uint32_t)e * 2654435761u) >> 21;
        static_assert(kNames == 1 << 11, "the hash has eleven bits");
        for (;;) {
            const int was = atomicCAS(&page[at], -1, e);
            if (was == -1 || was == e) return at;
            at = (at + 1) & (kNames - 1);
        }
    }
};

// A step's call (up to 1024 sequences that touch up to 1024 blocks in all) keeps a block per thread in registers from the first look at the
// tables to the last; what its phases exchange lies in LDS.  Others go over their blocks once per phase, with scratch in memory.
__global__ __launch_bounds__(kReserveThreads) void kv_reserve_kernel(KvPool p, KvTable t, const int32_t* len, const int32_t* cu, int32_t* pairs,
                                                                     int32_t* missing, KvReserveScratch w) {
    __shared__ int waves[kReserveWaves], ends[kReserveThreads], blocks[kReserveThreads], begun[kReserveThreads];
    __shared__ NameTable names;
    __shared__ KvRequest wanted[kReserveThreads];
    __shared__ int replaced[kReserveThreads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // ---- free pages, from the lowest on: a wave looks at 1024 neighbouring ones in a round of 16384
    constexpr int kRound = 16 * kReserveThreads;
    struct Pages {
        int4 names[4];
    };
    auto page_of = [&](int round, int u) { return round * kRound + wave * 1024 + u * 256 + lane * 4; };
    auto look = [&](int round) {
        Pages g;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int page = page_of(round, u);
            g.names[u] = make_int4(1, 1, 1, 1);
            if (page + 3 < p.n_pages) {
                g.names[u] = *reinterpret_cast<const int4*>(p.refs + page);
            } else {
                if (page < p.n_pages) g.names[u].x = p.refs[page];
                if (page + 1 < p.n_pages) g.names[u].y = p.refs[page + 1];
                if (page + 2 < p.n_pages) g.names[u].z = p.refs[page + 2];
            }
        }
        return g;
    };
    Pages pages = look(0);
    // serve(rank, page): gives the request of that rank the page; returns how many requests were served
    auto hand_out = [&](int requests, auto&& serve) {
        int served = 0;
        const int rounds = (p.n_pages + kRound - 1) / kRound;
        for (int round = 0; round < rounds && served < requests; ++round) {
            const Pages now = pages;
            if (round + 1 < rounds) pages = look(round + 1);
            int n[4], before[4], mine = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                n[u] = (now.names[u].x <= 0) + (now.names[u].y <= 0) + (now.names[u].z <= 0) + (now.names[u].w <= 0);
                const int up_to = wave_inclusive_scan(n[u]);
                before[u] = mine + up_to - n[u];
                mine += __builtin_amdgcn_readlane(up_to, 63);
            }
            __syncthreads();  // (`waves` may still be read)
            if (lane == 0) waves[wave] = mine;
            __syncthreads();
            int rank0 = served;
#pragma unroll
            for (int k = 0; k < kReserveWaves; ++k) {
                const int x = waves[k];
                rank0 += k < wave ? x : 0;
                served += x;
            }
            if (mine == 0 || rank0 >= requests) continue;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int here[4] = {now.names[u].x, now.names[u].y, now.names[u].z, now.names[u].w};
                int rank = rank0 + before[u];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (here[j] > 0) continue;
                    if (rank < requests) serve(rank, page_of(round, u) + j);
                    ++rank;
                }
            }
        }
        return min(served, requests);
    };
    auto entry = [&](int s, int b) { return t.at + (size_t)s * t.max_blocks + b; };
    // a sequence's first block, how many of its blocks lie inside the table, and how many behind it
    auto blocks_of = [&](int s, int& first, int& outside) {
        first = outside = 0;
        if (s >= t.n_seqs) return 0;
        const int L = length_of(len, s), rows = min(max(cu[s + 1] - cu[s], 0), kKvMaxLen);
        if (rows == 0) return 0;
        first = L / p.block;
        const int behind = (int)(((uint32_t)L + rows - 1) / p.block) + 1, n = max(0, min(behind, t.max_blocks) - first);
        outside = behind - first - n;
        return n;
    };
    // the sequence among a batch of 1024 (whose blocks end at ends[]) that a block belongs to
    auto owner = [&](int slot) {
        int lo = 0, hi = kReserveThreads - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (ends[mid] > slot) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    };
    for (int s = tid; s < t.n_seqs; s += kReserveThreads) pairs[2 * s] = pairs[2 * s + 1] = -1;
    if (t.n_seqs <= kReserveThreads) {
        for (int i = tid; i < kNames; i += kReserveThreads) names.page[i] = -1, names.first[i] = 0x7fffffff, names.writers[i] = 0;
        int first, outside, total;
        const int n = blocks_of(tid, first, outside), before = workgroup_scan(n, waves, total);
        ends[tid] = before + n;
        blocks[tid] = first - before;
        begun[tid] = tid < t.n_seqs && length_of(len, tid) % p.block != 0 ? first : -1;  // the block that holds tokens already
        __syncthreads();
        if (total <= kReserveThreads) {
            const bool there = tid < total;
            const int s = there ? owner(tid) : 0, b = blocks[s] + tid;
            const int e = there ? *entry(s, b) : -1;
            const int count = is_page(p, e) ? p.refs[e] : 0;
            const bool shared = is_page(p, e) && count > 1;
            bool need = there && !is_page(p, e);
            int place = 0;
            if (shared) {
                place = names.place(e);
                atomicMin(&names.first[place], s);
                atomicAdd(&names.writers[place], 1);
            }
            if (__syncthreads_or(shared) && shared) need = !(names.first[place] == s && count <= names.writers[place]);
            int requests;
            const int rank = workgroup_scan(need, waves, requests);
            if (need) wanted[rank] = KvRequest{s, b}, replaced[rank] = shared ? e : -1;
            int all_outside;
            workgroup_scan(min(outside, 1 << 20), waves, all_outside);  // (1024 threads' stay within 31 bits)
            const int served = hand_out(requests, [&](int rank, int page) {
                const KvRequest r = wanted[rank];
                const int old = replaced[rank];
                *entry(r.seq, r.block) = page;
                p.refs[page] = 1;
                if (old < 0) return;
                add_ref(p, old, -1);
                if (begun[r.seq] == r.block) pairs[2 * r.seq] = old, pairs[2 * r.seq + 1] = page;
            });
            if (tid == 0) *missing = requests - served + all_outside;
            return;
        }
    }
    // Every block that the call's rows touch, in order: f(sequence, block, whether there is one) by threads that take 1024 neighbouring ones at
    // a time (f is called by all threads together).  Returns how many blocks of this thread's sequences lie behind the table.
    auto each_block = [&](auto&& f) {
        int all_outside = 0;
        for (int s0 = 0; s0 < t.n_seqs; s0 += kReserveThreads) {
            int first, outside, total;
            const int n = blocks_of(s0 + tid, first, outside), before = workgroup_scan(n, waves, total);
            all_outside = min(all_outside + outside, 1 << 20);
            __syncthreads();  // (the arrays may still be read)
            ends[tid] = before + n;
            blocks[tid] = first - before;
            __syncthreads();
            for (int slot0 = 0; slot0 < total; slot0 += kReserveThreads) {
                const int slot = slot0 + tid, s = slot < total ? owner(slot) : 0;
                f(s0 + s, blocks[s] + slot, slot < total);
            }
        }
        return all_outside;
    };
    // pages with more than one name
    bool any = false;
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
                const int count = p.refs[e];
                need = count > 1 && !(load_agent(w.first + e) == s && count <= load_agent(w.writers + e));
            }
        }
        int all;
        const int rank = requests + workgroup_scan(need, waves, all);
        if (need && rank < p.n_pages) w.list[rank] = KvRequest{s, b};
        requests += all;
    });
    meet_in_memory();
    const int served = hand_out(requests, [&](int rank, int page) {
        const KvRequest r = w.list[rank];
        int32_t* at = entry(r.seq, r.block);
        const int old = *at, L = length_of(len, r.seq);
        *at = page;
        p.refs[page] = 1;
        if (!is_page(p, old)) return;
        add_ref(p, old, -1);
        if (r.block == L / p.block && L % p.block != 0) pairs[2 * r.seq] = old, pairs[2 * r.seq + 1] = page;
    });
    if (tid == 0) *missing = requests - served + outside;
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

// The same by one workgroup, for pools of up to kFewPages: eight pages per thread in registers, places in LDS.  us, one launch / three, with
// 1000 and 8000 entries: 100 pages 4.8 5.8 / 6.0, 2000 5.7 6.7 / 8.0, 8000 7.1 8.2 / 8.8; 32000 entries and 8000 pages 12.0 / 8.8.
__global__ __launch_bounds__(kReserveThreads) void kv_compact_few_kernel(KvPool p, KvTable t, int32_t* pairs, int n_pairs, int32_t* page_map) {
    __shared__ uint16_t place[kFewPages], high[kFewPages / 2], low[kFewPages / 2];
    __shared__ int waves[kReserveWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto page_of = [&](int u, int j) { return wave * 512 + u * 256 + lane * 4 + j; };
    int names[2][4], n[2], before[2], mine = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        int4 x = make_int4(0, 0, 0, 0);
        const int page = page_of(u, 0);
        if (page + 3 < p.n_pages) {
            x = *reinterpret_cast<const int4*>(p.refs + page);
        } else {
            if (page < p.n_pages) x.x = p.refs[page];
            if (page + 1 < p.n_pages) x.y = p.refs[page + 1];
            if (page + 2 < p.n_pages) x.z = p.refs[page + 2];
        }
        names[u][0] = x.x, names[u][1] = x.y, names[u][2] = x.z, names[u][3] = x.w;
        n[u] = (x.x > 0) + (x.y > 0) + (x.z > 0) + (x.w > 0);
        const int up_to = wave_inclusive_scan(n[u]);
        before[u] = mine + up_to - n[u];
        mine += __builtin_amdgcn_readlane(up_to, 63);
    }
    if (lane == 0) waves[wave] = mine;
    __syncthreads();
    int rank0 = 0, used = 0;
#pragma unroll
    for (int k = 0; k < kReserveWaves; ++k) {
        const int x = waves[k];
        rank0 += k < wave ? x : 0;
        used += x;
    }
    int below_mine = 0;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) below_mine += names[u][j] > 0 && page_of(u, j) < used;
    int below;
    workgroup_scan(below_mine, waves, below);
    const int moves = min(used - below, n_pairs);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        int rank = rank0 + before[u];  // used pages before the next one
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int page = page_of(u, j);
            if (page < p.n_pages) {
                place[page] = (uint16_t)page;
                if (names[u][j] > 0 && page >= used && used - 1 - rank < moves) high[used - 1 - rank] = (uint16_t)page;
                if (names[u][j] <= 0 && page < used && page - rank < moves) low[page - rank] = (uint16_t)page;
            }
            rank += names[u][j] > 0;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        int rank = rank0 + before[u];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int page = page_of(u, j), i = used - 1 - rank;
            if (page < p.n_pages && names[u][j] > 0 && page >= used && i < moves) {
                const int to = low[i];
                place[page] = (uint16_t)to;
                p.refs[to] = names[u][j];
                p.refs[page] = 0;
            }
            rank += names[u][j] > 0;
        }
    }
    for (int i = tid; i < n_pairs; i += kReserveThreads) {
        pairs[2 * i] = i < moves ? high[i] : -1;
        pairs[2 * i + 1] = i < moves ? low[i] : -1;
    }
    __syncthreads();
    for (int i = tid; i < p.n_pages; i += kReserveThreads) page_map[i] = place[i];
    const int entries = t.n_seqs * t.max_blocks;
#pragma unroll 4
    for (int i = tid; i < entries; i += kReserveThreads) {
        const int e = t.at[i], to = is_page(p, e) ? place[e] : e;
        if (to != e) t.at[i] = to;
    }
}

// ---- copy
// Bound by bytes, mostly those written (a page that goes to several places is read from L2: a workgroup's number mod 8 is its XCD, and pages
// mostly have a multiple of eight pieces).  Stores leave the caches to the sources.  us of a whole step of 128 beams with eight layers (82 MB
// written), of a fork and its end (252 MB), of packing and what is around it (472 MB), replayed: 45.8 69.3 174; with nontemporal stores alone
// 46.2 73 175.5, plain ones 6 10 5 more.  16 KB for a workgroup: 4 KB took 4 17 20 more, 8 KB 0 7 5, 32 KB 5 4 2.
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
    float* scales = is_v ? c.vs : c.ks;
    const float scale = scales[(size_t)from * a.heads + min(tid, a.heads - 1)];  // (by every piece, so that it needs no condition)
    if (at0 + kCopyBytes <= a.bytes) {  // (requests behind conditions of their own cost a quarter)
        constexpr int kPastCaches = 16 | 2;  // sc1 (written through) and nt
        const __amdgpu_buffer_rsrc_t to_page = __builtin_amdgcn_make_buffer_rsrc(dst + at0, 0, kCopyBytes, 0x00027000);
        u32x4 x[kCopyLoads];
#pragma unroll
        for (int i = 0; i < kCopyLoads; ++i) x[i] = *(const FLOE_GLOBAL u32x4*)(src + at0 + (i * kThreads + tid) * 16);
#pragma unroll
        for (int i = 0; i < kCopyLoads; ++i) __builtin_amdgcn_raw_buffer_store_b128(x[i], to_page, (i * kThreads + tid) * 16, 0, kPastCaches);
    } else {
        for (int at = at0 + tid * 16; at < a.bytes; at += kThreads * 16)
            __builtin_nontemporal_store(*(const FLOE_GLOBAL u32x4*)(src + at), (FLOE_GLOBAL u32x4*)(dst + at));
    }
    static_assert(kThreads >= 256, "a thread per head: a cache has up to 256");
    if (at0 == 0 && tid < a.heads) scales[(size_t)to * a.heads + tid] = scale;
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
    if (p.n_pages <= kFewPages && (int64_t)t.n_seqs * t.max_blocks <= kFewEntries) {
        kv_compact_few_kernel<<<dim3(1), dim3(kReserveThreads), 0, st>>>(p, t, pairs, n_pairs, page_map);
        return hipGetLastError();
    }
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
