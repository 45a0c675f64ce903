// Pages of the KV cache for gfx950: sequences that grow, shrink, fork and give their pages back, pages moved together, and the
// copies and appends that go with it (the cache that the serving side keeps under the rollouts, Sections 5.1 and 5.2).
//
// The state is four integer arrays: page_table with page_indptr (the paged attention's own), page_count (pages held by a
// sequence) and page_refs (table entries that name a page; 0 = free).  There is no free list: the i-th page that a call hands out
// is the i-th lowest free one, a prefix sum over page_refs, so equal states give equal tables whatever the device did before.
// A call is index work on a few hundred kilobytes at most, bound by launches and by the latency of dependent loads; the copies
// are bound by HBM.  Index work is done once per forward, copies once per layer: respec_pages_copy takes the lists that the
// others leave.
#include "respec_common.hpp"
#include "respec_tiles.hpp"

#include <algorithm>

namespace respec {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kRankThreads = 1024;
constexpr int kPagesPerBlock = 4 * kRankThreads;  // page_refs that a work-group ranks: four in a row per thread
// Up to here a work-group counts the pages before its own for itself (compaction of 16,384 pages 10.0 us with its enqueuing, of
// 16,385 in a launch more 11.9; at 32,768 the counting would take 14 us, the launch 5).
constexpr int kFewPages = 4 * kPagesPerBlock;
constexpr int kFewSequences = 32;             // up to here, and up to kPagesPerBlock pages, a resize is one launch
constexpr int32_t kKeep = INT32_MIN;          // a page that compaction neither moves nor fills
constexpr int32_t kMost = 1 << 30;            // pages, entries and moves lie below it: indices and strides are added in 32 bits

struct PageState {
    const int32_t *page_indptr;
    int32_t *page_table;
    int32_t *page_count;
    int32_t *kv_len;
    int32_t *page_refs;
    int32_t B, table_len, num_pages, page_shift;
};

// What the table of sequence b may hold: its first entry, its entries, and the pages it holds of them (all inside the buffers
// whatever the arrays hold).
struct Seq {
    int32_t e0, cap, count;
};
__device__ inline Seq seq_of(const PageState &p, int b) {
    Seq s;
    s.e0 = max(0, min(p.page_indptr[b], p.table_len));
    s.cap = max(0, min(p.page_indptr[b + 1], p.table_len) - s.e0);
    s.count = max(0, min(p.page_count[b], s.cap));
    return s;
}
__device__ inline bool is_page(const PageState &p, int32_t id) { return (uint32_t)id < (uint32_t)p.num_pages; }

// Inclusive sums over the threads of a work-group; `total` is everybody's.
template <int THREADS>
__device__ inline int block_scan(int x, int &total, int *lds /* [THREADS / 64] */) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int in_wave = wave_scan_add(x);
    if (lane == 63) lds[wave] = in_wave;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < THREADS / 64; ++w) {
        before += w < wave ? lds[w] : 0;
        total += lds[w];
    }
    __syncthreads();
    return before + in_wave;
}

template <int THREADS>
__device__ inline int block_sum_of(const int32_t *a, int n, int *lds) {
    int s = 0, total;
    for (int i = threadIdx.x; i < n; i += THREADS) s += a[i];
    block_scan<THREADS>(s, total, lds);
    return total;
}

// Free (LIVE: used) pages among the first n.
template <bool LIVE>
__device__ inline int block_count(const int32_t *refs, int n, int *lds) {
    int s = 0, total;
#pragma unroll 8
    for (int i = threadIdx.x; i < n; i += kRankThreads) s += LIVE ? refs[i] > 0 : refs[i] == 0;
    block_scan<kRankThreads>(s, total, lds);
    return total;
}

// ------------------------------------------------------------------------------------------ resize
struct ResizeParams {
    PageState s;
    const int32_t *want;
    int32_t *copy_src, *copy_dst, *missing;
    int32_t blocks;
    int32_t *block_free;  // [blocks] free pages of each block of page_refs
    int32_t *begin;       // [B] where a sequence's part of `fresh` begins
    int32_t *need;        // [B] how many it takes; bit 30: the first of them takes over a shared page's contents; bit 31: too many for its table
    int32_t *total_need;  // [1]
    int32_t *fresh;       // [num_pages] the free pages in order
};
constexpr int32_t kCopyBit = 1 << 30, kRefusedBit = INT32_MIN, kNeedMask = kCopyBit - 1;

// How many entries of a sequence from `from` up to `to` name a page that others name too.  They are the first of them: a child has all its parent's
// entries, a resize ends with a part that is the sequence's own and gives back from the end, so what two sequences have in common is
// the beginning of their tables.  None and all are seen at once, else the border is found by bisection.
__device__ inline int shared_from(const PageState &s, int32_t e0, int from, int to) {
    const auto is_shared = [&](int e) __attribute__((always_inline)) {
        const int32_t id = s.page_table[e0 + e];
        return is_page(s, id) && s.page_refs[id] > 1;
    };
    if (from >= to || !is_shared(from)) return 0;
    if (is_shared(to - 1)) return to - from;
    int last = from, own = to - 1;
    while (own - last > 1) {
        const int at = last + (own - last) / 2;
        if (is_shared(at)) last = at;
        else own = at;
    }
    return own - from;
}

// What sequence b needs, by the state before the call, as a word of `need`; `take`: the pages that it is counted for.  A sequence that grows gets
// a page of its own in the place of every shared one that it is about to write into, and needs the contents of the first if tokens lie in it.
__device__ inline int plan_of(const ResizeParams &p, int b, int &take) {
    const PageState &s = p.s;
    take = 0;
    if (p.want[b] < 0) return 0;
    const Seq q = seq_of(s, b);
    const int64_t pages = ((int64_t)p.want[b] + ((1 << s.page_shift) - 1)) >> s.page_shift;
    const int len = max(0, s.kv_len[b]);
    const int shared = p.want[b] > len ? shared_from(s, q.e0, len >> s.page_shift, (int)min(pages, (int64_t)q.count)) : 0;
    const bool copied = shared > 0 && (len & ((1 << s.page_shift) - 1)) != 0;
    const int64_t need = max((int64_t)0, pages - q.count) + shared;
    const int word = (int)min(need, (int64_t)kNeedMask) | (copied ? kCopyBit : 0);
    if (pages > q.cap) return word | kRefusedBit;
    take = (int)need;
    return word;
}
// (parts of page_table that overlap can ask for more than 2^31)
__device__ inline bool is_served(int word, int begin, int n_free) {
    const int need = word & kNeedMask;
    return (word & kRefusedBit) == 0 && (need == 0 || (begin >= 0 && (int64_t)begin + need <= n_free));
}

// Carries out the plan of sequence b, by the threads of a work-group or of a wave (`all_read`: everybody has read what one writes).  A page named by
// several sequences that let go of it in one call is counted down by each; a page handed out was free before the call, so no
// other sequence of the call names it.
template <int THREADS, typename F>
__device__ inline void resize_one(const ResizeParams &p, int b, int word, bool ok, const int32_t *fresh, int me, F &&all_read) {
    const PageState &s = p.s;
    const int want = p.want[b];
    const Seq q = seq_of(s, b);
    const int len = s.kv_len[b];
    all_read();
    if (me == 0) {
        p.missing[b] = want >= 0 && !ok ? word & kNeedMask : 0;
        p.copy_src[b] = p.copy_dst[b] = -1;
    }
    if (want < 0 || !ok) return;
    const int pages = (int)(((int64_t)want + ((1 << s.page_shift) - 1)) >> s.page_shift), at = max(0, len) >> s.page_shift;
    const int need = word & kNeedMask, shared = need - max(0, pages - q.count);  // (the shared ones come first)
    for (int e = pages + me; e < q.count; e += THREADS) {
        const int32_t id = s.page_table[q.e0 + e];
        if (is_page(s, id)) atomicSub(&s.page_refs[id], 1);
        s.page_table[q.e0 + e] = -1;
    }
    for (int i = me; i < need; i += THREADS) {
        const int32_t id = fresh[i];
        if (!is_page(s, id)) continue;  // (never, with tables as the header has them)
        int32_t *entry = &s.page_table[q.e0 + (i < shared ? at + i : q.count + i - shared)];
        if (i < shared) {
            const int32_t old = *entry;
            if (is_page(s, old)) atomicSub(&s.page_refs[old], 1);
            if (i == 0 && (word & kCopyBit) != 0) {
                p.copy_src[b] = old;
                p.copy_dst[b] = id;
            }
        }
        *entry = id;
        s.page_refs[id] = 1;
    }
    if (me == 0) {
        s.page_count[b] = pages;
        s.kv_len[b] = min(len, want);
    }
}

// The last work-group: what every sequence needs, by the state before the call.  The others: how many pages of a block are free,
// and (RANK) which these are in the order of all.
template <bool RANK>
__global__ __launch_bounds__(kRankThreads) void resize_plan_kernel(ResizeParams p) {
    __shared__ int lds[kRankThreads / 64];
    const PageState &s = p.s;
    int total;
    if ((int)blockIdx.x < p.blocks) {
        const int before = RANK ? block_count<false>(s.page_refs, blockIdx.x * kPagesPerBlock, lds) : 0;
        int is_free[4], n = 0;
        for (int i = 0; i < 4; ++i) {
            const int page = blockIdx.x * kPagesPerBlock + threadIdx.x * 4 + i;
            is_free[i] = page < s.num_pages && s.page_refs[page] == 0;
            n += is_free[i];
        }
        int rank = before + block_scan<kRankThreads>(n, total, lds) - n;
        if (threadIdx.x == 0) p.block_free[blockIdx.x] = total;
        if (RANK)
            for (int i = 0; i < 4; ++i)
                if (is_free[i]) p.fresh[rank++] = blockIdx.x * kPagesPerBlock + threadIdx.x * 4 + i;
        return;
    }
    int base = 0;
    for (int b0 = 0; b0 < s.B; b0 += kRankThreads) {
        const int b = b0 + threadIdx.x;
        int take = 0;
        const int word = b < s.B ? plan_of(p, b, take) : 0;
        const int to = block_scan<kRankThreads>(take, total, lds);
        if (b < s.B) {
            p.begin[b] = base + to - take;
            p.need[b] = word;
        }
        base += total;  // (at most the entries of page_table)
    }
    if (threadIdx.x == 0) *p.total_need = base;
}

// The free pages in order, as many as are needed, where the first launch did not rank them.
__global__ __launch_bounds__(kRankThreads) void resize_rank_kernel(ResizeParams p) {
    __shared__ int lds[kRankThreads / 64];
    const PageState &s = p.s;
    const int wanted = *p.total_need;
    if (wanted == 0) return;  // (uniform)
    const int before = block_sum_of<kRankThreads>(p.block_free, blockIdx.x, lds);
    if (before >= wanted) return;
    int is_free[4], n = 0, total;
    for (int i = 0; i < 4; ++i) {
        const int page = blockIdx.x * kPagesPerBlock + threadIdx.x * 4 + i;
        is_free[i] = page < s.num_pages && s.page_refs[page] == 0;
        n += is_free[i];
    }
    int rank = before + block_scan<kRankThreads>(n, total, lds) - n;
    for (int i = 0; i < 4; ++i)
        if (is_free[i]) p.fresh[rank++] = blockIdx.x * kPagesPerBlock + threadIdx.x * 4 + i;
}

// One work-group per sequence.  Both launches wait for a few loads that depend on one another: 3.1 and 3.7 us for 288 sequences.
__global__ __launch_bounds__(kThreads) void resize_apply_kernel(ResizeParams p) {
    __shared__ int lds[kThreads / 64];
    const int b = blockIdx.x, word = p.need[b], begin = p.begin[b];
    const int n_free = (word & kNeedMask) > 0 ? block_sum_of<kThreads>(p.block_free, p.blocks, lds) : 0;  // (uniform)
    resize_one<kThreads>(p, b, word, is_served(word, begin, n_free), p.fresh + begin, threadIdx.x, []() { __syncthreads(); });
}

// Few sequences and pages: all of it in one work-group, at the end a wave per sequence.  Replayed from a graph, a resize of 8 sequences in 4,096 pages
// takes 4.1 us, in two launches 6.5; of 32 sequences 5.4, and 6.5; of 64 7.3, and 6.4.  Enqueued one by one 7.0 and 9.3.
__global__ __launch_bounds__(kRankThreads) void resize_few_kernel(ResizeParams p) {
    __shared__ int lds[kRankThreads / 64];
    __shared__ int32_t fresh[kPagesPerBlock];
    __shared__ int begin[kFewSequences], need[kFewSequences];
    const PageState &s = p.s;
    int is_free[4], n = 0, n_free, total;
    for (int i = 0; i < 4; ++i) {
        const int page = threadIdx.x * 4 + i;
        is_free[i] = page < s.num_pages && s.page_refs[page] == 0;
        n += is_free[i];
    }
    int take = 0;
    const int word = (int)threadIdx.x < s.B ? plan_of(p, threadIdx.x, take) : 0;
    int rank = block_scan<kRankThreads>(n, n_free, lds) - n;
    for (int i = 0; i < 4; ++i)
        if (is_free[i]) fresh[rank++] = threadIdx.x * 4 + i;
    const int to = block_scan<kRankThreads>(take, total, lds);
    if ((int)threadIdx.x < s.B) {
        begin[threadIdx.x] = to - take;
        need[threadIdx.x] = word;
    }
    __syncthreads();  // (the state has been read as it was before the call)
    for (int b = threadIdx.x >> 6; b < s.B; b += kRankThreads / 64) {  // (uniform in a wave)
        const bool ok = is_served(need[b], begin[b], n_free);
        resize_one<64>(p, b, need[b], ok, fresh + (ok ? begin[b] : 0), threadIdx.x & 63, []() { __builtin_amdgcn_wave_barrier(); });
    }
}

// ------------------------------------------------------------------------------------------ fork
struct ForkParams {
    PageState s;
    const int32_t *parent;
    int32_t *missing;
};

// One work-group per sequence.  Only sequences with a parent are written, and a parent has none itself, so no work-group reads
// what another one writes (the counts of references aside, which are added to).  3.5 us for 256 children, dependent loads again.
__global__ __launch_bounds__(kThreads) void fork_kernel(ForkParams p) {
    const PageState &s = p.s;
    const int b = blockIdx.x, from = p.parent[b];
    if (from < 0) {
        if (threadIdx.x == 0) p.missing[b] = 0;
        return;
    }
    bool ok = from < s.B && from != b && p.parent[from] < 0;
    Seq q{}, f{};
    if (ok) {
        q = seq_of(s, b);
        f = seq_of(s, from);
        ok = q.count == 0 && f.count <= q.cap;
    }
    __syncthreads();  // (the count is read by everybody before one thread writes it)
    if (threadIdx.x == 0) p.missing[b] = ok ? 0 : -1;
    if (!ok) return;
    for (int e = threadIdx.x; e < f.count; e += kThreads) {
        const int32_t id = s.page_table[f.e0 + e];
        s.page_table[q.e0 + e] = id;
        if (is_page(s, id)) atomicAdd(&s.page_refs[id], 1);
    }
    if (threadIdx.x == 0) {
        s.page_count[b] = f.count;
        s.kv_len[b] = s.kv_len[from];
    }
}

// ------------------------------------------------------------------------------------------ compact
struct CompactParams {
    const int32_t *page_table, *page_refs;
    int32_t table_len, num_pages;
    int32_t *new_table, *new_refs;
    int32_t *copy_src, *copy_dst, *pages_end;
    int32_t max_moves, blocks;
    int32_t *block_live;  // [blocks]
    int32_t *n_live;      // [1] live pages
    int32_t *moves;       // [1] those behind the first n_live
    int32_t *role;        // [num_pages] n >= 0: the n-th highest of those; -1-n: the n-th lowest free page before them; kKeep
    int32_t *high, *hole; // [num_pages / 2 + 1] the pages with those roles
};

__global__ __launch_bounds__(kRankThreads) void compact_count_kernel(CompactParams p) {
    __shared__ int lds[kRankThreads / 64];
    int n = 0, total;
    for (int i = 0; i < 4; ++i) {
        const int page = blockIdx.x * kPagesPerBlock + threadIdx.x * 4 + i;
        n += page < p.num_pages && p.page_refs[page] > 0;
    }
    block_scan<kRankThreads>(n, total, lds);
    if (threadIdx.x == 0) p.block_live[blockIdx.x] = total;
}

// With n live pages in all, the m live ones behind the first n pages go to the m free ones among them.  Both numbers are the
// same, so a page's partner is known by its rank: highest live to lowest free, so that a bounded number of moves frees the end.
// COUNTED: a launch before has counted the blocks' live pages.
template <bool COUNTED>
__global__ __launch_bounds__(kRankThreads) void compact_rank_kernel(CompactParams p) {
    __shared__ int lds[kRankThreads / 64];
    const int before = COUNTED ? block_sum_of<kRankThreads>(p.block_live, blockIdx.x, lds)
                               : block_count<true>(p.page_refs, blockIdx.x * kPagesPerBlock, lds);
    const int n_live = COUNTED ? block_sum_of<kRankThreads>(p.block_live, p.blocks, lds) : block_count<true>(p.page_refs, p.num_pages, lds);
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.n_live = n_live;
    int live[4], n = 0, total;
    for (int i = 0; i < 4; ++i) {
        const int page = blockIdx.x * kPagesPerBlock + threadIdx.x * 4 + i;
        live[i] = page < p.num_pages && p.page_refs[page] > 0;
        n += live[i];
    }
    int rank = before + block_scan<kRankThreads>(n, total, lds) - n;  // live pages before this one
    for (int i = 0; i < 4; ++i) {
        const int page = blockIdx.x * kPagesPerBlock + threadIdx.x * 4 + i;
        if (page >= p.num_pages) break;
        int32_t role = kKeep;
        if (live[i] && page >= n_live) {
            role = n_live - 1 - rank;
            p.high[role] = page;
        } else if (!live[i] && page < n_live) {
            p.hole[page - rank] = page;
            role = -1 - (page - rank);
        }
        p.role[page] = role;
        rank += live[i];
        if (page == max(n_live, 1) - 1) *p.moves = n_live - (n_live > 0 ? rank : 0);
    }
}

// A thread per page, per table entry and per place of the lists.  (The three kernels take 4.6, 5.2 and 4.9 us for 256 sequences in 34,550 pages;
// the copies of a layer that follow 99.)
__global__ __launch_bounds__(kThreads) void compact_apply_kernel(CompactParams p) {
    const int moves = *p.moves, done = min(moves, p.max_moves);
    const int stride = gridDim.x * kThreads, first = blockIdx.x * kThreads + threadIdx.x;
    if (first == 0) *p.pages_end = moves <= p.max_moves ? *p.n_live : p.high[p.max_moves] + 1;
    for (int i = first; i < p.max_moves; i += stride) {
        p.copy_src[i] = i < done ? p.high[i] : -1;
        p.copy_dst[i] = i < done ? p.hole[i] : -1;
    }
    for (int page = first; page < p.num_pages; page += stride) {
        const int32_t role = p.role[page];
        if (role >= 0 && role < done) {
            const int32_t refs = p.page_refs[page];
            p.new_refs[p.hole[role]] = refs;
            p.new_refs[page] = 0;
        } else if (role >= 0 || role == kKeep || -1 - role >= done) {  // (a page that is filled is written by the one that goes there)
            p.new_refs[page] = p.page_refs[page];
        }
    }
    for (int e = first; e < p.table_len; e += stride) {
        int32_t id = p.page_table[e];
        if ((uint32_t)id < (uint32_t)p.num_pages) {
            const int32_t role = p.role[id];
            if (role >= 0 && role < done) id = p.hole[role];
        }
        p.new_table[e] = id;
    }
}

// ------------------------------------------------------------------------------------------ copy, append
struct CopyParams {
    char *k, *v;
    const int32_t *src, *dst;
    int32_t n, num_pages;
    int64_t page_bytes;
    int32_t chunks;  // of kChunk bytes in a page
};
constexpr int kChunk = kThreads * 16 * 4;  // a work-group's piece of a page: four 16-byte loads in flight per thread

// Loads and stores pass the caches by: a page is read and written once, 10,200 moves of 16-token pages of 16 KiB per pool take
// 209 us instead of 221 with ordinary ones (two layers, 1.06 GB read and written).
__global__ __launch_bounds__(kThreads) void copy_pages_kernel(CopyParams p) {
    const int64_t items = (int64_t)p.n * p.chunks * 2;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const int i = (int)(it / (2 * p.chunks)), rest = (int)(it % (2 * p.chunks));
        const int32_t src = p.src[i], dst = p.dst[i];
        if ((uint32_t)src >= (uint32_t)p.num_pages || (uint32_t)dst >= (uint32_t)p.num_pages || src == dst) continue;
        char *pool = rest & 1 ? p.v : p.k;
        const int64_t at = (int64_t)(rest >> 1) * kChunk;
        const char *from = pool + src * p.page_bytes + at;
        char *to = pool + dst * p.page_bytes + at;
        u32x4 x[4];
        for (int j = 0; j < 4; ++j) {
            const int64_t o = ((int64_t)j * kThreads + threadIdx.x) * 16;
            if (at + o < p.page_bytes) x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + o));
        }
        for (int j = 0; j < 4; ++j) {
            const int64_t o = ((int64_t)j * kThreads + threadIdx.x) * 16;
            if (at + o < p.page_bytes) __builtin_nontemporal_store(x[j], reinterpret_cast<u32x4 *>(to + o));
        }
    }
}

struct AppendParams {
    const char *k_new, *v_new;
    char *k, *v;
    const int32_t *q_indptr, *page_indptr, *page_table, *kv_len;
    int64_t ld_bytes;  // between tokens of k_new, v_new
    int32_t B, total_q, max_q, num_pages, table_len, page_shift, token_bytes;
};
constexpr int kAppendRows = 8;  // rows of a work-group

// Bound by memory: 4,096 tokens of 8 heads of 128 (33.6 MB read and written) take 7.7 us call after call, when the cache behind the L2s
// holds them, and 11.5 before an attention that displaces them; two loads in flight instead of eight 2 % more.
// A row's position follows from the length and the number of rows as they are given, whatever of them is left out: rows past max_q, and
// those whose position the sequence's pages do not have.
__global__ __launch_bounds__(kThreads) void append_kernel(AppendParams p) {
    Tile t;
    if (!find_tile(p.q_indptr, p.B, p.total_q, p.max_q, 1, kAppendRows, blockIdx.x, t)) return;
    const int e0 = max(0, min(p.page_indptr[t.b], p.table_len));
    const int pages = max(0, min(p.page_indptr[t.b + 1], p.table_len) - e0);
    const int64_t end = (int64_t)pages << p.page_shift;
    const int64_t pos0 = (int64_t)p.kv_len[t.b] - (min(p.q_indptr[t.b + 1], p.total_q) - t.q0);  // of row 0
    const int pieces = p.token_bytes / 16, rows = min(kAppendRows, t.R - t.index * kAppendRows);
    for (int i0 = threadIdx.x; i0 < rows * pieces; i0 += 4 * kThreads) {
        u32x4 a[4], c[4];
        int64_t to[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // (eight loads in flight: behind a store the next loads would wait, as the memory may be the same)
            to[j] = -1;
            const int i = i0 + j * kThreads, r = t.index * kAppendRows + i / pieces, piece = i % pieces;
            const int64_t pos = pos0 + r;
            if (i >= rows * pieces || pos < 0 || pos >= end) continue;
            const int32_t id = p.page_table[e0 + (pos >> p.page_shift)];
            if ((uint32_t)id >= (uint32_t)p.num_pages) continue;
            const int64_t from = (t.q0 + r) * p.ld_bytes + (int64_t)piece * 16;
            to[j] = (((int64_t)id << p.page_shift) + (pos & ((1 << p.page_shift) - 1))) * p.token_bytes + (int64_t)piece * 16;
            a[j] = *reinterpret_cast<const u32x4 *>(p.k_new + from);
            c[j] = *reinterpret_cast<const u32x4 *>(p.v_new + from);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (to[j] < 0) continue;
            *reinterpret_cast<u32x4 *>(p.k + to[j]) = a[j];
            *reinterpret_cast<u32x4 *>(p.v + to[j]) = c[j];
        }
    }
}

// ------------------------------------------------------------------------------------------ host side
int page_blocks(int32_t num_pages) { return (int)(((int64_t)num_pages + kPagesPerBlock - 1) / kPagesPerBlock); }

// 32-bit words: blocks, 64 single words, then for resize begin [B], need [B] and fresh [num_pages], for compact role
// [num_pages], high and hole [num_pages / 2 + 1] each.
size_t pages_words(int32_t B, int32_t num_pages) {
    const size_t resize = (size_t)2 * B + num_pages, compact = (size_t)num_pages + 2 * ((size_t)num_pages / 2 + 1);
    return (size_t)page_blocks(num_pages) + 64 + std::max(resize, compact);
}

respec_status_t check_state(const char *name, const void *a, const void *b, const void *c, const void *d, const void *e, int32_t B,
                            int32_t table_len, int32_t num_pages) {
    if (!a || !b || !c || !d || !e) return fail(RESPEC_ERR_INVALID_ARG, "%s: null pointer argument", name);
    if (B <= 0 || table_len <= 0 || num_pages <= 0)
        return fail(RESPEC_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d page_table_len=%d num_pages=%d)", name, B, table_len, num_pages);
    if (table_len >= kMost || num_pages >= kMost)
        return fail(RESPEC_ERR_UNSUPPORTED, "%s: page_table_len and num_pages must be below 2^30 (%d, %d)", name, table_len, num_pages);
    if (!grid_fits(B, kThreads)) return fail(RESPEC_ERR_UNSUPPORTED, "%s: too many sequences (%d)", name, B);
    return RESPEC_OK;
}

int shift_of(int32_t page_size) {
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0) return -1;
    return __builtin_ctz((unsigned)page_size);
}

respec_status_t check_workspace(const char *name, const void *workspace, size_t bytes, int32_t B, int32_t num_pages) {
    const size_t need = respec_pages_workspace_bytes(B, num_pages);
    if (!workspace || bytes < need || !aligned_to(workspace, 256))
        return fail(RESPEC_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) needed, got %zu", name, need, workspace ? bytes : (size_t)0);
    return RESPEC_OK;
}

respec_status_t launched(const char *name) {
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(RESPEC_ERR_HIP, "%s: launch failed: %s", name, hipGetErrorString(err));
    clear_error();
    return RESPEC_OK;
}

}  // namespace
}  // namespace respec

extern "C" {

size_t respec_pages_workspace_bytes(int32_t B, int32_t num_pages) {
    using namespace respec;
    if (B <= 0 || num_pages <= 0) return 0;
    return round_up(pages_words(B, num_pages) * sizeof(int32_t), 256);
}

respec_status_t respec_pages_resize(const int32_t *want_tokens, const int32_t *page_indptr, int32_t *page_table, int32_t *page_count,
                                    int32_t *kv_len, int32_t *page_refs, int32_t *copy_src, int32_t *copy_dst, int32_t *out_missing,
                                    int32_t B, int32_t page_table_len, int32_t num_pages, int32_t page_size, void *workspace,
                                    size_t workspace_bytes, void *hip_stream) {
    using namespace respec;
    respec_status_t st = check_state("pages_resize", page_indptr, page_table, page_count, kv_len, page_refs, B, page_table_len, num_pages);
    if (st != RESPEC_OK) return st;
    if (!want_tokens || !copy_src || !copy_dst || !out_missing) return fail(RESPEC_ERR_INVALID_ARG, "pages_resize: null pointer argument");
    const int shift = shift_of(page_size);
    if (shift < 0) return fail(RESPEC_ERR_UNSUPPORTED, "pages_resize: page size %d is not a power of two in [16, 1024]", page_size);
    if ((int64_t)page_table_len + B >= kCopyBit)
        return fail(RESPEC_ERR_UNSUPPORTED, "pages_resize: page_table_len + B must be below 2^30");
    st = check_workspace("pages_resize", workspace, workspace_bytes, B, num_pages);
    if (st != RESPEC_OK) return st;
    ResizeParams p{};
    p.s = {page_indptr, page_table, page_count, kv_len, page_refs, B, page_table_len, num_pages, shift};
    p.want = want_tokens;
    p.copy_src = copy_src;
    p.copy_dst = copy_dst;
    p.missing = out_missing;
    p.blocks = page_blocks(num_pages);
    p.total_need = static_cast<int32_t *>(workspace);
    p.block_free = p.total_need + 64;
    p.begin = p.block_free + p.blocks;
    p.need = p.begin + B;
    p.fresh = p.need + B;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (B <= kFewSequences && num_pages <= kPagesPerBlock) {
        hipLaunchKernelGGL(resize_few_kernel, dim3(1), dim3(kRankThreads), 0, stream, p);
        return launched("pages_resize");
    }
    if (num_pages <= kFewPages) {
        hipLaunchKernelGGL(resize_plan_kernel<true>, dim3(p.blocks + 1), dim3(kRankThreads), 0, stream, p);
    } else {
        hipLaunchKernelGGL(resize_plan_kernel<false>, dim3(p.blocks + 1), dim3(kRankThreads), 0, stream, p);
        hipLaunchKernelGGL(resize_rank_kernel, dim3(p.blocks), dim3(kRankThreads), 0, stream, p);
    }
    hipLaunchKernelGGL(resize_apply_kernel, dim3(B), dim3(kThreads), 0, stream, p);
    return launched("pages_resize");
}

respec_status_t respec_pages_fork(const int32_t *parent, const int32_t *page_indptr, int32_t *page_table, int32_t *page_count,
                                  int32_t *kv_len, int32_t *page_refs, int32_t *out_missing, int32_t B, int32_t page_table_len,
                                  int32_t num_pages, void *hip_stream) {
    using namespace respec;
    respec_status_t st = check_state("pages_fork", page_indptr, page_table, page_count, kv_len, page_refs, B, page_table_len, num_pages);
    if (st != RESPEC_OK) return st;
    if (!parent || !out_missing) return fail(RESPEC_ERR_INVALID_ARG, "pages_fork: null pointer argument");
    ForkParams p{};
    p.s = {page_indptr, page_table, page_count, kv_len, page_refs, B, page_table_len, num_pages, 0};
    p.parent = parent;
    p.missing = out_missing;
    hipLaunchKernelGGL(fork_kernel, dim3(B), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
    return launched("pages_fork");
}

respec_status_t respec_pages_compact(const int32_t *page_table, const int32_t *page_refs, int32_t *new_page_table, int32_t *new_page_refs,
                                     int32_t *copy_src, int32_t *copy_dst, int32_t *out_pages_end, int32_t page_table_len,
                                     int32_t num_pages, int32_t max_moves, void *workspace, size_t workspace_bytes, void *hip_stream) {
    using namespace respec;
    if (!page_table || !page_refs || !new_page_table || !new_page_refs || !copy_src || !copy_dst || !out_pages_end)
        return fail(RESPEC_ERR_INVALID_ARG, "pages_compact: null pointer argument");
    if (page_table_len <= 0 || num_pages <= 0 || max_moves <= 0)
        return fail(RESPEC_ERR_INVALID_ARG, "pages_compact: sizes must be positive (page_table_len=%d num_pages=%d max_moves=%d)", page_table_len,
                    num_pages, max_moves);
    if (page_table_len >= kMost || num_pages >= kMost || max_moves >= kMost)
        return fail(RESPEC_ERR_UNSUPPORTED, "pages_compact: page_table_len, num_pages and max_moves must be below 2^30 (%d, %d, %d)", page_table_len,
                    num_pages, max_moves);
    const respec_status_t st = check_workspace("pages_compact", workspace, workspace_bytes, 1, num_pages);
    if (st != RESPEC_OK) return st;
    CompactParams p{};
    p.page_table = page_table;
    p.page_refs = page_refs;
    p.table_len = page_table_len;
    p.num_pages = num_pages;
    p.new_table = new_page_table;
    p.new_refs = new_page_refs;
    p.copy_src = copy_src;
    p.copy_dst = copy_dst;
    p.pages_end = out_pages_end;
    p.max_moves = max_moves;
    p.blocks = page_blocks(num_pages);
    p.moves = static_cast<int32_t *>(workspace);
    p.n_live = p.moves + 1;
    p.block_live = p.moves + 64;
    p.role = p.block_live + p.blocks;
    p.high = p.role + num_pages;
    p.hole = p.high + num_pages / 2 + 1;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (num_pages <= kFewPages) {
        hipLaunchKernelGGL(compact_rank_kernel<false>, dim3(p.blocks), dim3(kRankThreads), 0, stream, p);
    } else {
        hipLaunchKernelGGL(compact_count_kernel, dim3(p.blocks), dim3(kRankThreads), 0, stream, p);
        hipLaunchKernelGGL(compact_rank_kernel<true>, dim3(p.blocks), dim3(kRankThreads), 0, stream, p);
    }
    const int64_t most = std::max({num_pages, page_table_len, max_moves});
    hipLaunchKernelGGL(compact_apply_kernel, dim3((unsigned)std::min<int64_t>((most + kThreads - 1) / kThreads, 1024)), dim3(kThreads), 0, stream, p);
    return launched("pages_compact");
}

respec_status_t respec_pages_copy(void *k_pages, void *v_pages, const int32_t *copy_src, const int32_t *copy_dst, int32_t n,
                                  int32_t num_pages, int32_t page_size, int32_t Hkv, int32_t D, respec_dtype_t dt, void *hip_stream) {
    using namespace respec;
    if (!k_pages || !v_pages || !copy_src || !copy_dst) return fail(RESPEC_ERR_INVALID_ARG, "pages_copy: null pointer argument");
    if (n <= 0 || num_pages <= 0 || page_size <= 0 || Hkv <= 0 || D <= 0)
        return fail(RESPEC_ERR_INVALID_ARG, "pages_copy: sizes must be positive (n=%d num_pages=%d page_size=%d Hkv=%d D=%d)", n, num_pages, page_size, Hkv, D);
    if (dt != RESPEC_F32 && dt != RESPEC_BF16) return fail(RESPEC_ERR_INVALID_ARG, "pages_copy: unknown dtype %d", (int)dt);
    if (shift_of(page_size) < 0) return fail(RESPEC_ERR_UNSUPPORTED, "pages_copy: page size %d is not a power of two in [16, 1024]", page_size);
    const int64_t token = (int64_t)Hkv * D * (dt == RESPEC_BF16 ? 2 : 4);
    if (token % 16 != 0 || token > (1 << 24)) return fail(RESPEC_ERR_UNSUPPORTED, "pages_copy: Hkv*D*sizeof(element) must be a multiple of 16 up to 2^24");
    if (!aligned_to(k_pages, 16) || !aligned_to(v_pages, 16)) return fail(RESPEC_ERR_INVALID_ARG, "pages_copy: k_pages and v_pages must be 16-byte aligned");
    CopyParams p{};
    p.k = static_cast<char *>(k_pages);
    p.v = static_cast<char *>(v_pages);
    p.src = copy_src;
    p.dst = copy_dst;
    p.n = n;
    p.num_pages = num_pages;
    p.page_bytes = token * page_size;
    p.chunks = (int32_t)((p.page_bytes + kChunk - 1) / kChunk);
    const int64_t items = (int64_t)n * p.chunks * 2;
    hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)std::min<int64_t>(items, 4096)), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
    return launched("pages_copy");
}

respec_status_t respec_append_paged(const void *k_new, const void *v_new, void *k_pages, void *v_pages, const int32_t *q_indptr,
                                    const int32_t *page_indptr, const int32_t *page_table, const int32_t *kv_len, int32_t B, int32_t total_q,
                                    int32_t max_q_per_seq, int32_t num_pages, int32_t page_table_len, int32_t page_size, int32_t Hkv,
                                    int32_t D, int64_t ld_new, respec_dtype_t dt, void *hip_stream) {
    using namespace respec;
    if (!k_new || !v_new || !k_pages || !v_pages || !q_indptr || !page_indptr || !page_table || !kv_len)
        return fail(RESPEC_ERR_INVALID_ARG, "append_paged: null pointer argument");
    if (B <= 0 || total_q <= 0 || max_q_per_seq <= 0 || num_pages <= 0 || page_table_len <= 0 || Hkv <= 0 || D <= 0)
        return fail(RESPEC_ERR_INVALID_ARG, "append_paged: sizes must be positive (B=%d total_q=%d)", B, total_q);
    if (dt != RESPEC_F32 && dt != RESPEC_BF16) return fail(RESPEC_ERR_INVALID_ARG, "append_paged: unknown dtype %d", (int)dt);
    const int shift = shift_of(page_size);
    if (shift < 0) return fail(RESPEC_ERR_UNSUPPORTED, "append_paged: page size %d is not a power of two in [16, 1024]", page_size);
    const int64_t esz = dt == RESPEC_BF16 ? 2 : 4, token = (int64_t)Hkv * D * esz;
    if (ld_new < (int64_t)Hkv * D) return fail(RESPEC_ERR_INVALID_ARG, "append_paged: token stride smaller than Hkv*D");
    if (token % 16 != 0 || token > (1 << 24) || (ld_new * esz) % 16 != 0)
        return fail(RESPEC_ERR_UNSUPPORTED, "append_paged: tokens must be whole 16-byte pieces (Hkv*D up to 2^24 bytes, ld_new)");
    if (!aligned_to(k_pages, 16) || !aligned_to(v_pages, 16) || !aligned_to(k_new, 16) || !aligned_to(v_new, 16))
        return fail(RESPEC_ERR_INVALID_ARG, "append_paged: data pointers must be 16-byte aligned");
    AppendParams p{};
    p.k_new = static_cast<const char *>(k_new);
    p.v_new = static_cast<const char *>(v_new);
    p.k = static_cast<char *>(k_pages);
    p.v = static_cast<char *>(v_pages);
    p.q_indptr = q_indptr;
    p.page_indptr = page_indptr;
    p.page_table = page_table;
    p.kv_len = kv_len;
    p.ld_bytes = ld_new * esz;
    p.B = B;
    p.total_q = total_q;
    p.max_q = max_q_per_seq;
    p.num_pages = num_pages;
    p.table_len = page_table_len;
    p.page_shift = shift;
    p.token_bytes = (int32_t)token;
    const int64_t grid = tiles_bound(B, total_q, max_q_per_seq, 1, kAppendRows);
    if (!grid_fits(grid, kThreads)) return fail(RESPEC_ERR_UNSUPPORTED, "append_paged: too many rows");
    hipLaunchKernelGGL(append_kernel, dim3((unsigned)grid), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
    return launched("append_paged");
}

}  // extern "C"
