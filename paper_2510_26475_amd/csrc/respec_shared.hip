// Verify attention for gfx950 over a paged cache whose sequences share their beginnings, in the cache's type or over a cache of 8 bits.
//
// The responses of a rollout group hold the pages of their prompt together.  The rows of all of them see all the keys that they share, so
// these are a product of many rows (128 to a work-group) with each key and value read once, and only what a sequence holds by itself is read for its own few
// rows.  With (m, l, o) the running maximum, sum and unnormalised output of a part of the keys, the parts are joined by
//     m = max m_i,   l = sum_i l_i 2^(m_i - m),   o = sum_i o_i 2^(m_i - m) / l.
// A work-group does one of the two kinds of work, in one launch: the shared part keeps the matrix cores busy, the other one the memory, and a compute unit
// holds two work-groups.  Both kinds form a flat list of tiles that is cut into even ranges, so every work-group has as much to do whatever the lengths
// are (what beginning and ending with a sequence takes is counted); a range that ends inside a sequence leaves a part, and a second kernel joins the parts in a fixed order.
//
// Products as in the prompt attention: S^T = K Q^T with 32 packed rows (G heads of a KV head to a row) as a wave's columns, the probabilities of a lane's column
// the B operand of O^T = V^T P^T, exponents against a running maximum that moves only where it grows by more than 2^8.
#include "respec_common.hpp"
#include "respec_quantised.hpp"
#include "respec_tiles.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

namespace respec {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef s16x4 __attribute__((address_space(3))) *LdsTr;
typedef __attribute__((address_space(3))) void *LdsTo;
typedef const __attribute__((address_space(1))) void *GlobalFrom;
typedef const __attribute__((address_space(4))) int32_t *ConstInts;  // (read through the scalar cache; nothing writes it meanwhile)

constexpr float kRescaleSlack = 8.f;  // log2 units
constexpr int kWorkGroups = 512;      // two for each compute unit
constexpr int kThreads = 256, kPrepThreads = 512;
constexpr int kPrepGroups = 8;        // work-groups that share the jobs out, each with a plan of its own
constexpr int kColumns = 32;          // of a wave
constexpr int kBlock = 4 * kColumns;  // columns of a work-group over shared keys
constexpr int kJobs = 4 * kWorkGroups;  // one for each wave, or for the waves that share one
constexpr int kFewSeqs = 1024, kFewGroups = 256;  // whose plan is made in LDS

struct SeqPlan {
    int64_t base;              // its place in the list of own work
    int32_t q0, R, L, e0;      // first row, rows, tokens, first entry of page_table
    int32_t shared, group;     // tokens that its group reads for it; -1: none
    int32_t tiles, before;     // tiles of its own; sequences before it that have some
};
struct SeqGroup {              // of a sequence's group, for the join
    int64_t base;
    int32_t q0, rows, key_tiles, pad;
};
struct GroupPlan {
    int64_t base;              // its place in the list of shared work
    int32_t q0, rows, shared, e0;
    int32_t key_tiles, blocks; // tiles of keys, blocks of columns
    int32_t first, end;        // its sequences
    int32_t before, pad;       // blocks before its
};
enum Kind { kNone = 0, kShared = 1, kOwn = 2 };
struct Job {                   // a range: where it begins and all that its work-group (own work: its wave) needs for that
    uint64_t key;              // of the sizes that the plan was made for
    int32_t kind, range, tiles;
    int32_t outer, item, tile, block, pad;
    SeqPlan s;
    GroupPlan g;
};
// A flat list of `total` places cut into n even ranges: the first `more` of them have one more than the others.  Every sequence with keys of its own and every
// block of columns has a place for each of its tiles, and `head` before them for what it takes to begin and to end with it.
struct Cut {
    int64_t total, each;
    int32_t n, more;
};
struct Totals {
    Cut own, shared;
    int64_t own_step, shared_step;  // places of an outer step of own work; of a head of shared work
    int32_t shared_wgs, own_head, shared_head, pad;  // heads: as the cuts were made with them
    uint64_t key;                   // of the sizes that the plan was made for
};

struct SharedParams {
    const char *q, *k, *v;
    const uint8_t *k_scale, *v_scale;
    const int32_t *q_indptr, *page_indptr, *page_table, *kv_len, *group_indptr, *shared_len;
    const uint64_t *tree_mask;
    char *out;
    float *lse;
    int32_t B, groups, total_q, max_q, max_kv, num_pages, table_len, page_shift;
    int32_t Hq, Hkv, G;
    int32_t heads_wg, parts_wg, col_waves;  // KV heads, parts of the keys and column tiles that a work-group's four waves handle (own work)
    int32_t outer;                          // (head group, column block) pairs of own work
    uint32_t g_mul, g_shift;                // of a division by G
    uint32_t q_and, q_xor;                  // on the bits of q: a negative scale is taken out of it, a zero one makes it zero
    float scale2;                           // |sm_scale| * log2(e)
    int32_t own_head, shared_head;          // places before the tiles of a sequence and of a block (the plan's; the join goes by what the plan holds)
    float own_cost;                         // of a work-group's tile of own keys, against one of shared keys
    int32_t max_ranges, min_tiles;
    uint64_t key;
    SeqPlan *seq;
    SeqGroup *seq_grp;
    GroupPlan *grp;
    Job *jobs;
    Totals *totals;
    // Parts of ranges' ends, and those that are a row's only one of their kind ([total_q * Hq]): outputs, and four words with maximum, sum and the outputs' unit.
    char *own_o, *shared_o, *own_whole_o, *shared_whole_o;
    float *own_ml, *shared_ml, *own_whole_ml, *shared_whole_ml;
};

// x / G by a product: with s = ceil(log2 G) and g_mul = floor(2^32 (2^s - G) / G) + 1 this is exact for every x below 2^32.
__device__ inline int by_g(const SharedParams &p, int x) {
    const uint32_t t = __umulhi((uint32_t)x, p.g_mul);
    return p.G == 1 ? x : (int)((t + (((uint32_t)x - t) >> 1)) >> (p.g_shift - 1));
}

enum Pool { kF32 = 0, kBf16 = 1, kE4m3 = 2 };

template <Pool POOL, int D>
struct Shape {
    static constexpr bool kHalf = POOL != kF32;                   // products in bf16
    static constexpr int kSize = kHalf ? 2 : 4, kPoolSize = POOL == kE4m3 ? 1 : kSize;
    static constexpr int kRowBytes = D * kSize;                   // of a key in LDS
    static constexpr int kPieces = kRowBytes / 16;                // of 16 bytes in it
    static constexpr int kPoolPieces = D * kPoolSize / 16;        // of a key in the pool
    static constexpr int kLoadKeys = 64 / kPoolPieces;            // keys of a wave's load
    static constexpr int kDTiles = D / 32;
    static constexpr int kOwnKeys = 32, kOwnLoads = kOwnKeys / kLoadKeys;
    static constexpr int kCodeBytes = kOwnKeys * D;               // 8 bits: K or V of a tile as it is, two of each to a wave, and its scales
    static constexpr int kOwnBytes = POOL == kE4m3 ? 4 * kCodeBytes + 2 * kOwnKeys * 4 : 2 * kOwnKeys * kRowBytes;
    static constexpr int kSharedKeys = kHalf ? 64 : 32, kWaveKeys = kSharedKeys / 4;
    static constexpr int kSharedLoads = kWaveKeys / kLoadKeys, kSharedBytes = 2 * kSharedKeys * kRowBytes;
    static constexpr int kPlaces = kHalf ? 5 : 4;                 // for K or V of a tile of shared keys in LDS: three (two) of K, two of V
    static constexpr int kTileBytes = 2 * kOwnKeys * D * kPoolSize;  // of K and V as they are in the pool
    static constexpr int kPairedRing = 4, kPairedHeads = 2;       // 8 bits: tiles in LDS where waves share them; KV heads at most
    static constexpr int kPairedBytes = POOL == kE4m3 ? kPairedHeads * kPairedRing * (kTileBytes + 64 + 16) + 4 * 2 * kOwnKeys * 4 : 0;
    static constexpr int most(int a, int b) { return a > b ? a : b; }
    static constexpr int kLdsBytes = most(most(4 * kOwnBytes, kPlaces * kSharedBytes / 2), kPairedBytes);
    static_assert(kSharedLoads >= 1 && 16 % kLoadKeys == 0, "a wave's load lies in one page");
};

// Where a 16-byte piece of a key's row lies in the row, so that the lanes that read together meet different banks: K is read as
// one piece per key (sixteen keys at a time), V (bf16) as four keys by 64 bytes, V (fp32) along a row.
template <bool HALF, int D>
__device__ inline int k_piece(int key, int c) {
    if constexpr (HALF && D == 64) return c ^ ((key >> 1) & 7);
    else return c ^ (key & 15);
}
template <bool HALF, int D>
__device__ inline int v_piece(int key, int c) {
    if constexpr (!HALF) return c;
    else if constexpr (D == 128) return c ^ ((key & 3) << 2);
    else return c ^ (((key >> 1) & 1) << 2);
}

__device__ inline float max_of_halves(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float sum_of_halves(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ inline void wave_sync() {  // (a wave's LDS operations run in order: only the compiler is held back)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ------------------------------------------------------------------------------------------ the plan
__device__ __attribute__((always_inline)) inline int64_t begin_of(const Cut &c, int r) { return r * c.each + min(r, c.more); }
// a / b for a below 2^52: the quotient in floating point is off by one at most.
__device__ inline int64_t quotient(int64_t a, int64_t b) {
    if ((a | b) >> 31 == 0) return (uint32_t)a / (uint32_t)b;
    int64_t x = (int64_t)((double)a / (double)b);
    x -= x * b > a;
    return x + ((x + 1) * b <= a);
}
__device__ inline Cut make_cut(int64_t total, int ranges) {
    Cut c{};
    c.total = total;
    c.n = (int)min(total, (int64_t)ranges);
    c.each = c.n == 0 ? 0 : quotient(total, c.n);
    c.more = c.n == 0 ? 0 : (int)(total - c.each * c.n);
    return c;
}
__device__ inline int range_of(const Cut &c, int64_t f) {  // the range that tile f lies in
    const int64_t longer = c.more * (c.each + 1);
    return (int)(f < longer ? quotient(f, c.each + 1) : c.more + quotient(f - longer, c.each));
}

// Exclusive sums over the threads: of x below 2^31 and y below 2^58, as parts whose sums over the threads fit 32 bits, and of two whose sums do.
struct Sums {
    int64_t x, y;
    int32_t u, w;
};
__device__ inline void block_scan(int x, int64_t y, int u, int w, Sums &before, Sums &all, int (*lds)[8]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int v[7] = {x & 8191, x >> 13, (int)(y & 0xfffff), (int)(y >> 20 & 0xfffff), (int)(y >> 40), u, w};
    int sum[7], total[7] = {};
#pragma unroll
    for (int i = 0; i < 7; ++i) sum[i] = wave_scan_add(v[i]);
    if (lane == 63)
#pragma unroll
        for (int i = 0; i < 7; ++i) lds[wave][i] = sum[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 7; ++i) sum[i] -= v[i];
#pragma unroll
    for (int k = 0; k < kPrepThreads / 64; ++k)
#pragma unroll
        for (int i = 0; i < 7; ++i) {
            sum[i] += k < wave ? lds[k][i] : 0;
            total[i] += lds[k][i];
        }
    __syncthreads();
    auto joined = [](const int (&t)[7]) __attribute__((always_inline)) {
        return Sums{t[0] + ((int64_t)t[1] << 13), t[2] + ((int64_t)t[3] << 20) + ((int64_t)t[4] << 40), t[5], t[6]};
    };
    before = joined(sum);
    all = joined(total);
}

// Where places f[0] and f[1] of the flat list are: the last items whose bases are not past them.  (Both at once: each step of one waits for LDS.)
template <typename Item>
__device__ inline void find_items(const Item *items, int n, const int64_t (&f)[2], int (&at)[2]) {
    int end[2] = {n, n};
    at[0] = at[1] = 0;
    for (int span = n; span > 1; span = (span + 1) / 2)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int mid = (at[i] + end[i]) / 2;
            if (items[mid].base <= f[i]) at[i] = mid;
            else end[i] = mid;
        }
}

template <typename T>
__device__ inline void copy_plan(T &to, const T &from) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 8); ++i) reinterpret_cast<uint64_t *>(&to)[i] = reinterpret_cast<const uint64_t *>(&from)[i];
}

// What each sequence and group has to do, and where the ranges begin.  Up to kFewSeqs sequences every work-group makes the plan for itself, in LDS, and all
// share the jobs out and write the plan down; for more there is one work-group.  Latency: with 256 sequences in 32 groups the index arrays take 1.3 us, the groups 1.1,
// the sums 1.3, the cut 0.7 and the jobs 1.
template <int SHARED_KEYS, bool FEW>
__global__ __launch_bounds__(kPrepThreads) void shared_prep_kernel(SharedParams p) {
    __shared__ int lds[kPrepThreads / 64][8];
    __shared__ SeqPlan lds_seq[FEW ? kFewSeqs : 1];
    __shared__ GroupPlan lds_grp[FEW ? kFewGroups : 1];
    SeqPlan *const seq = FEW ? lds_seq : p.seq;
    GroupPlan *const grp = FEW ? lds_grp : p.grp;
    // A group shares what all its members hold before their new tokens.
    bool mixed = false;  // offsets that decrease: sequences could be in two groups, so nothing is shared
    auto group = [&](int g) __attribute__((always_inline)) {
        const int from = p.group_indptr[g], to = p.group_indptr[g + 1], first = max(0, min(from, p.B)), end = max(first, min(to, p.B));
        mixed |= to < from;
        GroupPlan t{};
        t.first = first;
        t.end = end;
        t.shared = end - first < 2 ? 0 : max(0, p.shared_len[g]);
        return t;
    };
    GroupPlan mine{};  // (on its way while the sequences are)
    if ((int)threadIdx.x < p.groups) mine = group(threadIdx.x);
    for (int b = threadIdx.x; b < p.B; b += kPrepThreads) {
        SeqPlan s{};
        const int q0 = p.q_indptr[b], q1 = p.q_indptr[b + 1], e0 = p.page_indptr[b], e1 = p.page_indptr[b + 1], length = p.kv_len[b];
        s.q0 = max(0, min(q0, p.total_q));
        s.R = max(0, min(max(0, min(q1, p.total_q)) - s.q0, p.max_q));
        s.e0 = max(0, min(e0, p.table_len));
        const int64_t held = max(0, max(0, min(e1, p.table_len)) - s.e0);
        s.L = (int)max((int64_t)0, min(min((int64_t)length, held << p.page_shift), (int64_t)p.max_kv));
        s.group = -1;
        seq[b] = s;
    }
    if ((int)threadIdx.x < p.groups) grp[threadIdx.x] = mine;
    for (int g = threadIdx.x + kPrepThreads; g < p.groups; g += kPrepThreads) grp[g] = group(g);
    const bool none = __syncthreads_or(mixed);
    auto group_of = [&](int b) __attribute__((always_inline)) {  // the last one that begins at or before b, if b is in it
        int at = 0;
        for (int end = p.groups; end - at > 1;) {
            const int mid = (at + end) / 2;
            if (grp[mid].first <= b) at = mid;
            else end = mid;
        }
        return p.groups > 0 && grp[at].first <= b && b < grp[at].end ? at : -1;
    };
    for (int b = threadIdx.x; b < p.B && p.groups > 0; b += kPrepThreads) {
        const int g = group_of(b);
        seq[b].group = g;
        if (g >= 0) __hip_atomic_fetch_min(&grp[g].shared, max(0, seq[b].L - seq[b].R), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    __syncthreads();
    for (int g = threadIdx.x; g < p.groups; g += kPrepThreads) {
        const int shared = __hip_atomic_load(&grp[g].shared, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP), first = grp[g].first, end = grp[g].end;
        GroupPlan t{};
        t.first = first;
        t.end = end;
        if (shared > 0 && !none) {
            t.q0 = seq[first].q0;
            t.rows = max(0, seq[end - 1].q0 + seq[end - 1].R - t.q0);
            t.e0 = seq[first].e0;
            t.shared = t.rows > 0 ? shared : 0;
            t.key_tiles = (t.shared + SHARED_KEYS - 1) / SHARED_KEYS;
            t.blocks = (int)(((int64_t)t.rows * p.G + kBlock - 1) / kBlock);
        }
        grp[g] = t;
    }
    __syncthreads();
    Sums done{};  // tiles of own and of shared keys, sequences with own ones, blocks
    for (int i0 = 0; i0 < max(p.B, p.groups); i0 += kPrepThreads) {
        const int i = i0 + threadIdx.x;
        int tiles = 0, blocks = 0;
        int64_t shared_tiles = 0;
        if (i < p.B) {
            SeqPlan s = seq[i];
            s.shared = s.group < 0 ? 0 : grp[s.group].shared;
            seq[i].shared = s.shared;
            if (s.R > 0 && s.L > s.shared) tiles = (int)(((int64_t)s.L + 31) / 32) - s.shared / 32;
        }
        if (i < p.groups) {
            blocks = grp[i].blocks;
            shared_tiles = (int64_t)grp[i].key_tiles * blocks;
        }
        Sums before, all;
        block_scan(tiles, shared_tiles, tiles > 0, blocks, before, all, lds);
        if (i < p.B) {
            seq[i].before = done.u + before.u;
            seq[i].base = done.x + before.x + (int64_t)p.own_head * seq[i].before;
            seq[i].tiles = tiles;
        }
        if (i < p.groups) {
            grp[i].before = done.w + before.w;
            grp[i].base = done.y + before.y + (int64_t)p.shared_head * grp[i].before;
        }
        done = Sums{done.x + all.x, done.y + all.y, done.u + all.u, done.w + all.w};
    }
    const int64_t own = done.x + (int64_t)p.own_head * done.u, shared = done.y + (int64_t)p.shared_head * done.w;
    // Work-groups for each kind by what its tiles cost, whole eights of them (the XCDs take turns).
    Totals t{};
    t.own_step = own;
    t.shared_step = shared;
    const int64_t all_own = own * p.outer, all_shared = shared * p.Hkv;
    if (all_shared > 0) {
        const float cost_s = (float)all_shared, cost_o = (float)all_own / p.parts_wg * p.own_cost;
        const int even = (int)(kWorkGroups / 8 * (cost_s / (cost_s + cost_o)) + 0.5f) * 8;
        t.shared_wgs = all_own > 0 ? max(8, min(even, kWorkGroups - 8)) : kWorkGroups;
    }
    t.shared = make_cut(all_shared, min(t.shared_wgs, p.max_ranges));
    // (at least a few tiles to a range: parts have to be joined)
    t.own = make_cut(all_own, (int)min((int64_t)min((kWorkGroups - t.shared_wgs) * p.parts_wg, p.max_ranges), (all_own + p.min_tiles - 1) / p.min_tiles));
    t.own_head = p.own_head;
    t.shared_head = p.shared_head;
    t.key = p.key;
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.totals = t;
    __syncthreads();
    // (wave after wave of all work-groups: the first one by itself needs 2 us for 512 jobs)
    const int turn = (threadIdx.x / 64 * gridDim.x + blockIdx.x) * 64 + threadIdx.x % 64;
    for (int j = turn; j < kWorkGroups * p.parts_wg; j += gridDim.x * kPrepThreads) {
        const int wg = j / p.parts_wg;
        Job &job = p.jobs[wg * 4 + j - wg * p.parts_wg];
        int kind = kNone;
        if (wg < t.shared_wgs) {
            // consecutive ranges, which read the same keys for other columns, on one XCD (work-groups go to the XCDs in turn)
            const int r = wg % 8 * (t.shared_wgs / 8) + wg / 8;
            if (r < t.shared.n) {
                // The range's first place and the one behind its last: where they are, and how many tiles come before them.
                int64_t f[2] = {begin_of(t.shared, r), begin_of(t.shared, r + 1)}, before[2];
                int outer[2], item[2], block[2], tile[2];
                for (int i = 0; i < 2; ++i) {
                    outer[i] = (int)quotient(f[i], shared);
                    f[i] -= outer[i] * shared;
                }
                find_items(grp, p.groups, f, item);
                for (int i = 0; i < 2; ++i) {
                    const int64_t in = f[i] - grp[item[i]].base;
                    const int key_tiles = grp[item[i]].key_tiles, places = key_tiles + p.shared_head;
                    block[i] = (int)quotient(in, places);
                    tile[i] = max(0, (int)(in - (int64_t)block[i] * places) - p.shared_head);
                    before[i] = outer[i] * done.y + grp[item[i]].base - (int64_t)p.shared_head * grp[item[i]].before + (int64_t)block[i] * key_tiles + tile[i];
                }
                if (before[1] > before[0]) kind = kShared;
                job.range = r;
                job.tiles = (int)(before[1] - before[0]);
                job.outer = outer[0];
                job.item = item[0];
                job.block = block[0];
                job.tile = tile[0];
                copy_plan(job.g, grp[item[0]]);
            }
        } else {
            const int r = j - t.shared_wgs * p.parts_wg;
            if (r < t.own.n) {
                int64_t f[2] = {begin_of(t.own, r), begin_of(t.own, r + 1)}, before[2];
                int outer[2], item[2], tile[2];
                for (int i = 0; i < 2; ++i) {
                    outer[i] = (int)quotient(f[i], own);
                    f[i] -= outer[i] * own;
                }
                find_items(seq, p.B, f, item);
                for (int i = 0; i < 2; ++i) {
                    tile[i] = max(0, (int)(f[i] - seq[item[i]].base) - p.own_head);
                    before[i] = outer[i] * done.x + seq[item[i]].base - (int64_t)p.own_head * seq[item[i]].before + tile[i];
                }
                if (before[1] > before[0]) kind = kOwn;
                job.range = r;
                job.tiles = (int)(before[1] - before[0]);
                job.outer = outer[0];
                job.item = item[0];
                job.tile = tile[0];
                copy_plan(job.s, seq[item[0]]);
            }
        }
        job.kind = kind;
        job.key = p.key;
    }
    const int last = gridDim.x * kPrepThreads - 1 - turn;  // (from the other end: waves without jobs)
    for (int b = last; b < p.B; b += gridDim.x * kPrepThreads) {
        if (FEW) copy_plan(p.seq[b], seq[b]);
        const int g = seq[b].group;
        if (g >= 0) copy_plan(p.seq_grp[b], SeqGroup{grp[g].base, grp[g].q0, grp[g].rows, grp[g].key_tiles, 0});
    }
    if (FEW)
        for (int g = last; g < p.groups; g += gridDim.x * kPrepThreads) copy_plan(p.grp[g], grp[g]);
}

// ------------------------------------------------------------------------------------------ what both kinds of work do
template <Pool POOL, int D>
struct State {  // of a wave's 32 columns
    using S = Shape<POOL, D>;
    floatx16 o[S::kDTiles];  // O^T: d = 32 d-tile + 8 (x / 4) + 4 half + x % 4
    float m, ref, l;
    u32x4 qf[S::kPieces / 2];
    __device__ void clear() {
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
            for (int x = 0; x < 16; ++x) o[d][x] = 0.f;
        m = -INFINITY;
        ref = l = 0.f;
    }
    // The scores of a tile to probabilities: the maximum moves where it grows by more than 2^8, the sum is theirs before any rounding.
    __device__ __attribute__((always_inline)) inline void exponentials(const SharedParams &p, floatx16 &s) {
        float top = s[0];
#pragma unroll
        for (int x = 1; x < 16; ++x) top = fmaxf(top, s[x]);
        rescale(p, top);
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            s[x] = __builtin_amdgcn_exp2f(fmaf(s[x], p.scale2, -ref));
            l += s[x];
        }
    }
    __device__ __attribute__((always_inline)) inline void rescale(const SharedParams &p, float top) {  // with the largest score that this lane has
        top = max_of_halves(top) * p.scale2;
        if (__ballot(top > m + kRescaleSlack) == 0) return;  // (m = -inf: any finite score)
        const float m_new = top > m + kRescaleSlack ? top : m;
        const float f = m == m_new ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        ref = m_new == -INFINITY ? 0.f : m_new;
        l *= f;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
            for (int x = 0; x < 16; ++x) o[d][x] *= f;
    }
    // Q^T as the B operand: a lane's column is its row, its contraction slots the pieces 2x + half of the row (CODES: as sixteen codes of K lie together,
    // the pieces 4 (x / 2) + 2 half + x % 2).
    template <bool CODES = false>
    __device__ void load_q(const SharedParams &p, int64_t row, int head, int half) {
        const char *from = p.q + (row * p.Hq + head) * (int64_t)S::kRowBytes + half * (CODES ? 32 : 16);
#pragma unroll
        for (int x = 0; x < S::kPieces / 2; ++x) qf[x] = *reinterpret_cast<const u32x4 *>(from + (CODES ? x / 2 * 64 + x % 2 * 16 : x * 32));
    }
    __device__ void sign_q(const SharedParams &p) {  // (apart: the loads are not waited for where they are requested)
#pragma unroll
        for (int x = 0; x < S::kPieces / 2; ++x)
            for (int w = 0; w < 4; ++w) qf[x][w] = (qf[x][w] & p.q_and) ^ p.q_xor;
    }
};

// A tile of 32 keys in LDS (K at `k`, V at `v`): the scores, masked by mask(), into the state.
template <Pool POOL, int D, typename Mask>
__device__ __attribute__((always_inline)) inline void attend(const SharedParams &p, State<POOL, D> &st, const char *lds, int k, int v, int half, int col, Mask &&mask) {
    using S = Shape<POOL, D>;
    // The place of a piece within its row is an exclusive or, so the x-th pair of pieces of K lies at k_at ^ 32 x and the d-th tile of V at v_at ^ 64 d.
    int k_at = k + col * S::kRowBytes + k_piece<S::kHalf, D>(col, half) * 16;
    asm volatile("" : "+v"(k_at));  // (the addresses that follow from it would not fit beside the tiles in flight)
    floatx16 s, other;  // (a second chain of products: a wave by itself waits for each)
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = other[x] = 0.f;
#pragma unroll
    for (int x = 0; x < S::kPieces / 2; ++x) {
        const u32x4 a = *reinterpret_cast<const u32x4 *>(lds + (k_at ^ (32 * x)));
        if constexpr (S::kHalf) {
            floatx16 &to = x % 2 == 0 ? s : other;
            to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, st.qf[x]), to, 0, 0, 0);
        } else {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                floatx16 &to = y % 2 == 0 ? s : other;
                to = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[y]), __uint_as_float(st.qf[x][y]), to, 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] += other[x];
    mask(s);
    st.exponentials(p, s);
    if constexpr (S::kHalf) {
        // V by transposing reads: sixteen lanes address four keys by sixteen d and receive one d of the four keys each.
        const int lane = half * 32 + col, i16 = lane & 15, v_key = half * 4 + (i16 >> 2), d0 = ((lane & 16) + 4 * (i16 & 3)) * 2;
        int v_at = v + v_key * S::kRowBytes + v_piece<true, D>(v_key, d0 >> 4) * 16 + (d0 & 15);
        asm volatile("" : "+v"(v_at));
#pragma unroll
        for (int g = 0; g < 2; ++g) {  // sixteen keys at a time: slot j is key 8 (j / 4) + 4 half + j % 4 of them; their probabilities rounded to bf16
            u32x4 pf;
#pragma unroll
            for (int j = 0; j < 4; ++j) pf[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{s[g * 8 + 2 * j], s[g * 8 + 2 * j + 1]}, bf16x2));
#pragma unroll
            for (int d = 0; d < S::kDTiles; ++d) {
                s16x4 vt[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) vt[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTr)(lds + (v_at ^ (64 * d)) + (g * 16 + j * 8) * S::kRowBytes));
                st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(vt[0], vt[1], 0, 1, 2, 3, 4, 5, 6, 7)),
                                                                  __builtin_bit_cast(bf16x8, pf), st.o[d], 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const int key = 8 * (x / 4) + 4 * half + x % 4;
#pragma unroll
            for (int d = 0; d < S::kDTiles; ++d)
                st.o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float *>(lds + v + key * S::kRowBytes + (d * 32 + col) * 4), s[x], st.o[d], 0, 0, 0);
        }
    }
}

// Where sixteen keys of a sequence lie that begin at key n (a multiple of eight), all in one page: keys past the last one are the last one's, as they are
// never seen.  The entry of the page table is asked for a step before it is needed (waited for at once: 96 sequences of 256 to 8,192 tokens with trees of seven rows at
// 40/8 heads over 8 bits 181 us, 162 so).
struct Run {
    int32_t entry, slot, left;  // slot: of the first; left: keys behind it
    __device__ __attribute__((always_inline)) inline Run(const SharedParams &p, int e0, int n, int last) {
        n = min(n, last);
        entry = ((ConstInts)p.page_table)[e0 + (n >> p.page_shift)];
        slot = n & ((1 << p.page_shift) - 1);
        left = last - n;
    }
    __device__ int64_t page(const SharedParams &p) const { return max(0, min(entry, p.num_pages - 1)); }
    __device__ int64_t row(const SharedParams &p, int h) const { return ((page(p) << p.page_shift) + slot) * p.Hkv + h; }
    __device__ int64_t scale(const SharedParams &p, int h) const { return ((page(p) * p.Hkv + h) << p.page_shift) + slot; }
};
struct Runs {  // of 32 keys
    Run a, b;
    __device__ __attribute__((always_inline)) inline Runs(const SharedParams &p, int e0, int n, int last) : a(p, e0, n, last), b(p, e0, n + 16, last) {}
    __device__ const Run &operator[](int i) const { return i == 0 ? a : b; }
};

// A wave's 32 keys on their way from the pools through registers into LDS (fp32 and bf16).  What differs between lanes is a 32-bit offset.
template <Pool POOL, int D>
struct Mover {
    using S = Shape<POOL, D>;
    static constexpr int kLoads = S::kOwnLoads, kRun = 16 / S::kLoadKeys;
    u32x4 k[kLoads], v[kLoads];
    __device__ __attribute__((always_inline)) inline void load(const SharedParams &p, const Runs &runs, int h, int lane) {
        const int my_key = lane / S::kPoolPieces;
        const uint32_t piece = (uint32_t)(lane % S::kPoolPieces) * 16, token = (uint32_t)p.Hkv * D * S::kPoolSize;
#pragma unroll
        for (int run = 0; run < kLoads / kRun; ++run) {
            const Run &r = runs[run];
            const char *kp = p.k + r.row(p, h) * (D * S::kPoolSize), *vp = p.v + r.row(p, h) * (D * S::kPoolSize);
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                const uint32_t off = (uint32_t)min(j * S::kLoadKeys + my_key, r.left) * token + piece;
                k[run * kRun + j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kp + off));  // (read once)
                v[run * kRun + j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(vp + off));
            }
        }
    }
    // Into a tile.  SIFT: some row does not see all of these keys.  A product would carry a value of V that is not finite to it all the same, so such values
    // count as zero here (they are added at the end to the rows that see them), as do all of keys outside [begin, end).
    template <bool SIFT>
    __device__ __attribute__((always_inline)) inline bool put(char *kt, char *vt, int lane, int n0, int begin, int end) {
        asm volatile("" : "+v"(lane));  // (as in attend)
        const int my_key = lane / S::kPoolPieces, piece = lane % S::kPoolPieces, row = my_key * S::kRowBytes;
        // (kLoadKeys keys on, the place of a piece of K differs by an exclusive or and that of V not at all)
        const int k_at = row + k_piece<S::kHalf, D>(my_key, piece) * 16, v_at = row + v_piece<S::kHalf, D>(my_key, piece) * 16;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            u32x4 b = v[i];
            if constexpr (SIFT) {
                const int n = n0 + i * S::kLoadKeys + my_key;
                const bool none = n < begin || n >= end;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const bool hi = (b[w] & 0x7f800000u) == 0x7f800000u, lo = S::kHalf && (b[w] & 0x7f80u) == 0x7f80u;
                    bad |= (hi || lo) && !none;
                    b[w] &= none ? 0u : (hi ? (S::kHalf ? 0xffffu : 0u) : ~0u) & (lo ? 0xffff0000u : ~0u);
                }
            }
            constexpr int kStep = S::kLoadKeys * S::kRowBytes;
            *reinterpret_cast<u32x4 *>(kt + (k_at ^ (k_piece<S::kHalf, D>(i * S::kLoadKeys, 0) * 16)) + i * kStep) = k[i];
            *reinterpret_cast<u32x4 *>(vt + v_at + i * kStep) = b;
        }
        return bad;
    }
};

enum RowType { kOutRow, kPartRow, kWideRow };  // the output (bf16), a part (fp16), a part whose numbers lie too far apart for fp16 (bf16)
// A wave's column times `factor` to `to`, a row of D; nullptr: there is no such column.  The halves of the wave trade four of
// eight d each, so that a lane writes sixteen bytes (through LDS, eight columns at a time: 96 sequences with trees of seven rows 163 us, 152 so).
template <Pool POOL, int D, RowType ROW>
__device__ __attribute__((always_inline)) inline void write_row(const State<POOL, D> &st, float factor, char *to, int half) {
    using S = Shape<POOL, D>;
#pragma unroll
    for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
        for (int x = 0; x < 16; x += 8) {
            uint32_t y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const floatx2 a = {st.o[d][x + 2 * j] * factor, st.o[d][x + 2 * j + 1] * factor};
                y[j] = ROW != kPartRow ? __builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2)) : __builtin_bit_cast(uint32_t, __builtin_convertvector(a, halfx2));
            }
            const auto lo = __builtin_amdgcn_permlane32_swap(y[0], y[2], false, false), hi = __builtin_amdgcn_permlane32_swap(y[1], y[3], false, false);
            const u32x4 z = {lo[0], hi[0], lo[1], hi[1]};
            u32x4 *const at = reinterpret_cast<u32x4 *>(to + (32 * d + 2 * x + 8 * half) * 2);
            if (to && ROW == kOutRow) __builtin_nontemporal_store(z, at);
            else if (to) *at = z;  // (read soon)
        }
}

// A wave's column as a part: to row `to` of `ml` its maximum, its sum, the unit of its output and whether that is a wide row, to row `to` of `o` the unnormalised
// output (negative: there is no such column).  Outputs of bf16 products are written in fp16, in a unit that puts the largest of a row between 2^14 and 2^15:
// the rounding is at most 2^-11 of each number down to 2^-29 of the largest, against 2^-8 of the probabilities before and of the result after (half
// the bytes: 256 sequences of 512 to 4,096 tokens at 28/4 heads over 8 bits leave 20 MB).  A row with a smaller number that is not zero (channels of V
// that far apart; by cancellation one row in a million) is written in bf16, as it is: 2^-8 of each number.  What is not finite stays so.  Returns the wide
// rows, a bit for each column.
template <Pool POOL, int D>
__device__ __attribute__((always_inline)) inline uint32_t write_part(const State<POOL, D> &st, float l, char *o, float *ml, int half, int64_t to) {
    using S = Shape<POOL, D>;
    float factor = 1.f, unit = 1.f;
    uint32_t wide = 0;
    if constexpr (S::kHalf) {
        float top = 0.f;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; ++x) top = fmaxf(top, fabsf(st.o[d][x]));
        if (__ballot(top == INFINITY) != 0) {  // (NaN is passed over, infinities are here)
            top = 0.f;
#pragma unroll
            for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
                for (int x = 0; x < 16; ++x) top = fmaxf(top, fabsf(st.o[d][x]) < INFINITY ? fabsf(st.o[d][x]) : 0.f);
        }
        const int e = max(-97, (int)(__float_as_uint(max_of_halves(top)) >> 23) - 126);  // top < 2^e, 128 at most
        factor = __uint_as_float((uint32_t)(142 - e) << 23);
        unit = __uint_as_float((uint32_t)(112 + e) << 23);
        // The smallest magnitude that is not zero, by its bits (twice them less one: zero is the largest), against 2^-14 units, where fp16 begins to lose bits.
        uint32_t least = ~0u;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; ++x) least = min(least, (__float_as_uint(st.o[d][x]) << 1) - 1);
        const uint64_t lanes = __ballot(least < ((uint32_t)(98 + e) << 24) - 1);
        wide = (uint32_t)lanes | (uint32_t)(lanes >> 32);
    }
    const bool mine = wide >> (threadIdx.x & 31) & 1;
    if (half == 0 && to >= 0) *reinterpret_cast<floatx4 *>(ml + to * 4) = floatx4{st.m, l, mine ? 1.f : unit, mine ? 1.f : 0.f};
    if constexpr (S::kHalf) {
        char *const row = to < 0 ? nullptr : o + to * (D * 2);
        write_row<POOL, D, kPartRow>(st, factor, mine ? nullptr : row, half);
        if (wide != 0) write_row<POOL, D, kWideRow>(st, 1.f, mine ? row : nullptr, half);
    } else if (to >= 0) {
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; x += 4)
                *reinterpret_cast<floatx4 *>(o + (to * D + d * 32 + 2 * x + 4 * half) * 4) = floatx4{st.o[d][x], st.o[d][x + 1], st.o[d][x + 2], st.o[d][x + 3]};
    }
    return wide;
}

// One of two buffers of a workspace.  (Chosen by the pointers themselves, the compiler keeps both in scratch and reads the one that is meant.)
template <typename T>
__device__ inline T *either(bool first, T *a, T *b) { return b + (first ? a - b : 0); }

// ------------------------------------------------------------------------------------------ keys that a group shares
// f(0), f(1) ... f(N-1), each with its number as a type.
template <int N, typename F, int... I>
__device__ __attribute__((always_inline)) inline void each_of(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __attribute__((always_inline)) inline void each(F &&f) {
    each_of<N>(f, std::make_integer_sequence<int, N>{});
}

// K or V of a tile of shared keys on its way from the pool into LDS: each wave moves a quarter of the keys, which lie in one page.  bf16: straight into
// LDS, each lane asking for the piece that belongs where its sixteen bytes land.  8 bits: K through registers and V through LDS as it is (`to`), where each lane
// finds again what it has asked for, to be turned into bf16; there would not be registers for both.  fp32: through registers.
template <Pool POOL, int D, bool V>
struct Stage {
    using S = Shape<POOL, D>;
    static constexpr bool kDirect = POOL == kBf16, kRaw = POOL == kE4m3 && V;
    static constexpr int kLoads = S::kSharedLoads;
    u32x4 x[kDirect || kRaw ? 1 : kLoads];
    uint32_t scale;  // of the wave's key `lane`
    __device__ __attribute__((always_inline)) inline void load(const SharedParams &p, const GroupPlan &g, int h, int tile, int wave, int lane, char *to) {
        const Run r(p, g.e0, tile * S::kSharedKeys + wave * S::kWaveKeys, g.shared - 1);
        const char *from = (V ? p.v : p.k) + r.row(p, h) * (D * S::kPoolSize);
        const uint32_t token = (uint32_t)p.Hkv * D * S::kPoolSize;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int in_wave = i * S::kLoadKeys + lane / S::kPoolPieces, key = wave * S::kWaveKeys + in_wave, at = lane % S::kPoolPieces;
            const int piece = !kDirect ? at : V ? v_piece<S::kHalf, D>(key, at) : k_piece<S::kHalf, D>(key, at);  // (an exclusive or: its own inverse)
            const char *mine = from + ((uint32_t)min(in_wave, r.left) * token + (uint32_t)piece * 16);
            if constexpr (kDirect)
                __builtin_amdgcn_global_load_lds((GlobalFrom)mine, (LdsTo)(to + (wave * S::kWaveKeys + i * S::kLoadKeys) * S::kRowBytes), 16, 0, 0);
            else if constexpr (kRaw)
                __builtin_amdgcn_global_load_lds((GlobalFrom)mine, (LdsTo)(to + (wave * kLoads + i) * 1024), 16, 0, 0);
            else
                x[i] = *reinterpret_cast<const u32x4 *>(mine);
        }
        if constexpr (kRaw) asm volatile("" ::: "memory");  // (the scale is asked for last: put() goes by that)
        if constexpr (POOL == kE4m3) scale = (V ? p.v_scale : p.k_scale)[r.scale(p, h) + min(lane % S::kWaveKeys, r.left)];
    }
    // What load() has asked for, into the tile (straight ones are there).  Of V, what lies past the shared keys is zero: `end` keys of the tile are shared.
    __device__ __attribute__((always_inline)) inline void put(char *tile, int wave, int lane, int end, const char *raw = nullptr) const {
        asm volatile("" : "+v"(lane));
        // (loads come back in order: with the scale, which was asked for last, the codes are there)
        if constexpr (kRaw) asm volatile("" ::"v"(scale) : "memory");
        if constexpr (kDirect) {
            if (V && end < S::kSharedKeys)
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
                    if (wave * S::kWaveKeys + i * S::kLoadKeys + lane / S::kPieces >= end)
                        *reinterpret_cast<u32x4 *>(tile + (wave * S::kWaveKeys + i * S::kLoadKeys) * S::kRowBytes + lane * 16) = u32x4{0, 0, 0, 0};
        } else {
            constexpr int kOut = POOL == kE4m3 ? 2 : 1;
            const int my_key = wave * S::kWaveKeys + lane / S::kPoolPieces, piece = lane % S::kPoolPieces * kOut;
            const int at = my_key * S::kRowBytes + (V ? v_piece<S::kHalf, D>(my_key, piece) : k_piece<S::kHalf, D>(my_key, piece)) * 16;
            u32x4 mine[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if constexpr (kRaw) mine[i] = *reinterpret_cast<const u32x4 *>(raw + (wave * kLoads + i) * 1024 + lane * 16);
                else mine[i] = x[i];
            }
            // (read, before the next straight load into `raw` is asked for: nothing else holds that back)
            if constexpr (kRaw)
#pragma unroll
                for (int i = 0; i < kLoads; ++i) asm volatile("" : "+v"(mine[i]) : : "memory");
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                u32x4 a[kOut];
                if constexpr (POOL == kE4m3) {
                    const u32x4 codes = mine[i];
                    const float step = scale_of(__shfl((int)scale, i * S::kLoadKeys + lane / S::kPoolPieces));
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        uint32_t lo, hi;
                        values_of(codes[w], step, lo, hi);
                        a[w / 2][w % 2 * 2] = lo;
                        a[w / 2][w % 2 * 2 + 1] = hi;
                    }
                } else {
                    a[0] = mine[i];
                }
                if (V && end < S::kSharedKeys) {
#pragma unroll
                    for (int y = 0; y < kOut; ++y)
                        for (int w = 0; w < 4; ++w) a[y][w] &= my_key + i * S::kLoadKeys < end ? ~0u : 0u;
                }
#pragma unroll
                for (int y = 0; y < kOut; ++y)
                    *reinterpret_cast<u32x4 *>(tile + (at ^ (V ? 16 * y : k_piece<S::kHalf, D>(i * S::kLoadKeys, y) * 16)) + i * S::kLoadKeys * S::kRowBytes) = a[y];
            }
        }
    }
};

// Scores of keys past the shared ones are masked.
template <int NB>
__device__ __attribute__((always_inline)) inline void mask_past(floatx16 (&s)[NB], int n0, int half, int end) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int x = 0; x < 16; ++x)
            if (n0 + b * 32 + 8 * (x / 4) + 4 * half + x % 4 >= end) s[b][x] = -INFINITY;
}

// All but the `kLeft` loads that the wave has asked for last are there.
template <int kLeft>
__device__ __attribute__((always_inline)) inline void wait_for() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (kLeft & 15) | (kLeft >> 4) << 14);  // vmcnt(kLeft)
    asm volatile("" ::: "memory");
}
// The waves of the work-group meet: what they have written to LDS is there, and all but those loads.
template <int kLeft>
__device__ __attribute__((always_inline)) inline void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (kLeft & 15) | (kLeft >> 4) << 14);  // vmcnt(kLeft) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// fp32: tiles t0 .. t1-1 one after the other, one of them read while the next is on its way.
template <int D>
__device__ __attribute__((always_inline)) inline void shared_tiles(const SharedParams &p, char *lds, const GroupPlan &g, int h, int t0, int t1, bool active, State<kF32, D> &st) {
    using S = Shape<kF32, D>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    Stage<kF32, D, false> k;
    Stage<kF32, D, true> v;
    k.load(p, g, h, t0, wave, lane, nullptr);
    v.load(p, g, h, t0, wave, lane, nullptr);
    st.sign_q(p);
    for (int t = t0; t < t1; ++t) {
        const int at = (t - t0) % 2 * S::kSharedBytes, n0 = t * S::kSharedKeys;
        k.put(lds + at, wave, lane, S::kSharedKeys);
        v.put(lds + at + S::kSharedBytes / 2, wave, lane, g.shared - n0);
        if (t + 1 < t1) {
            k.load(p, g, h, t + 1, wave, lane, nullptr);
            v.load(p, g, h, t + 1, wave, lane, nullptr);
        }
        __syncthreads();  // (this tile is there, and the one before the last has been read)
        if (active)
            attend(p, st, lds, at, at + S::kSharedBytes / 2, half, col, [&](floatx16 &s) __attribute__((always_inline)) {
                if (n0 + S::kSharedKeys <= g.shared) return;
                floatx16 x[1] = {s};
                mask_past(x, n0, half, g.shared);
                s = x[0];
            });
    }
    __syncthreads();
}

// bf16 products: the scores of tile t+1 are multiplied while the exponentials of tile t are computed, so step t reads K of t+1 and V of t.  LDS holds
// three (8 bits: two) tiles of K and two of V.  bf16: step t asks for K of t+3 and V of t+1, whose places were read a step before; K is waited for two
// steps on.  8 bits: it puts K of t+2 and V of t+1 in their places and asks for K of t+4 and V of t+3 (a step is shorter than the memory's latency).  Written in the
// order it is to run in: a product, an LDS read kReads products before its use, and a share of the rest.
template <Pool POOL, int D>
__device__ __attribute__((always_inline)) inline void shared_tiles(const SharedParams &p, char *lds, const GroupPlan &g, int h, int t0, int t1, bool active, State<POOL, D> &st) {
    using S = Shape<POOL, D>;
    typedef Stage<POOL, D, false> StageK;
    typedef Stage<POOL, D, true> StageV;
    constexpr bool kDirect = StageK::kDirect;
    constexpr int kTile = S::kSharedBytes / 2, kBlocks = S::kSharedKeys / 32;  // of K or V; of 32 keys
    constexpr int kRing = kDirect ? 3 : 2, kV = kRing * kTile;                 // places of K; where V's begin
    constexpr int kFirst = kBlocks * S::kPieces / 2, kSecond = 2 * kBlocks * S::kDTiles, kReads = 4;
    constexpr int kPairs = 16 * kBlocks / 2, kEarly = kPairs * 5 / 8;          // pairs of probabilities; those along with the first products
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int last_tile = t1 - 1;
    StageK k[kDirect ? 1 : 2];
    StageV v[kDirect ? 1 : 2];
    char *const raw = lds + 4 * kTile;  // two tiles of codes of V
    auto v_end = [&](int t) __attribute__((always_inline)) { return g.shared - t * S::kSharedKeys; };
    // Tiles t0, t0+1 (and t0+2) of K and t0 (and t0+1) of V.
    auto fetch_k = [&](StageK &x, int t, char *to) __attribute__((always_inline)) { x.load(p, g, h, min(t, last_tile), wave, lane, to); };  // (past the last tile: not read)
    auto fetch_v = [&](StageV &x, int t, char *to) __attribute__((always_inline)) { x.load(p, g, h, min(t, last_tile), wave, lane, to); };
    if constexpr (kDirect) {
        fetch_k(k[0], t0, lds);
        fetch_v(v[0], t0, lds + kV);
        fetch_k(k[0], t0 + 1, lds + kTile);
        fetch_k(k[0], t0 + 2, lds + 2 * kTile);
    } else {
        fetch_k(k[0], t0, nullptr);
        fetch_v(v[0], t0, raw);
        fetch_k(k[1], t0 + 1, nullptr);
        fetch_v(v[1], t0 + 1, raw + kTile / 2);
        k[0].put(lds, wave, lane, S::kSharedKeys);
        fetch_k(k[0], t0 + 2, nullptr);
        v[0].put(lds + kV, wave, lane, v_end(t0), raw);
        fetch_v(v[0], t0 + 2, raw);
        k[1].put(lds + kTile, wave, lane, S::kSharedKeys);
        fetch_k(k[1], t0 + 3, nullptr);
    }
    // The place of a piece within its row is an exclusive or, so the x-th pair of pieces of K lies at k_at ^ 32 x and the d-th tile of V at v_at ^ 64 d.
    int k_at = col * S::kRowBytes + k_piece<true, D>(col, half) * 16;
    const int i16 = lane & 15, v_key = half * 4 + (i16 >> 2), d0 = ((lane & 16) + 4 * (i16 & 3)) * 2;
    int v_at = kV + v_key * S::kRowBytes + v_piece<true, D>(v_key, d0 >> 4) * 16 + (d0 & 15);

    auto largest = [&](const floatx16(&s)[kBlocks]) __attribute__((always_inline)) {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int x = b == 0; x < 16; ++x) top = fmaxf(top, s[b][x]);
        return top;
    };
    // Two probabilities of sixteen keys' B operand, the n-th pair of all: slot j is key 8 (j / 4) + 4 half + j % 4 of them.  Rounded to bf16 for the
    // second product (2^-8 each at most, averaging over the keys); the sum is that of the unrounded ones.
    auto pair = [&](auto n_, const floatx16(&s)[kBlocks], u32x4(&pf)[2 * kBlocks]) __attribute__((always_inline)) {
        constexpr int n = decltype(n_)::value, i = n / 4, j = n % 4 * 2;
        const float a = __builtin_amdgcn_exp2f(fmaf(s[i / 2][i % 2 * 8 + j], p.scale2, -st.ref));
        const float c = __builtin_amdgcn_exp2f(fmaf(s[i / 2][i % 2 * 8 + j + 1], p.scale2, -st.ref));
        st.l += a;
        st.l += c;
        asm volatile("" : "+v"(st.l));  // (added now: later, the sixteen pairs would have to be kept)
        pf[i][j / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, c}, bf16x2));
    };
    auto read_v = [&](int i, int d, int tile) __attribute__((always_inline)) {
        s16x4 vt[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) vt[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTr)(lds + (v_at ^ (64 * d)) + (tile + (i * 16 + j * 8) * S::kRowBytes)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(vt[0], vt[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // Step t (not the last), whose scores are in s with their maximum taken into account.  KPLACE, VPLACE: (t - t0) modulo the places of K and of V.
    auto step = [&](auto k_place, auto v_place, int t, floatx16(&s)[kBlocks], floatx16(&next)[kBlocks]) __attribute__((always_inline)) {
        constexpr int kPlace = decltype(k_place)::value, vPlace = decltype(v_place)::value;
        char *const v_to = lds + kV + (vPlace ^ 1) * kTile;
        if constexpr (kDirect) {
            fetch_v(v[0], t + 1, v_to);
            fetch_k(k[0], t + 3, lds + kPlace * kTile);
        }
        asm volatile("" : "+v"(k_at), "+v"(v_at));  // (the addresses that follow from them would not fit beside the tiles)
        if (active) {
            __builtin_amdgcn_sched_barrier(0);
            bf16x8 ahead[kReads];
            u32x4 pf[2 * kBlocks];
            auto read = [&](auto i_) __attribute__((always_inline)) {
                constexpr int i = decltype(i_)::value;
                if constexpr (i < kFirst) {
                    constexpr int b = i % kBlocks, x = i / kBlocks;
                    ahead[i % kReads] = *reinterpret_cast<const bf16x8 *>(lds + (k_at ^ (32 * x)) + ((kPlace + 1) % kRing * kTile + b * 32 * S::kRowBytes));
                } else if constexpr (i < kFirst + kSecond) {
                    ahead[i % kReads] = read_v((i - kFirst) / S::kDTiles, (i - kFirst) % S::kDTiles, vPlace * kTile);
                }
            };
            float top = -INFINITY;
            each<kReads>([&](auto i) __attribute__((always_inline)) { read(i); });
            __builtin_amdgcn_sched_barrier(0);
            each<kFirst + kSecond>([&](auto i_) __attribute__((always_inline)) {
                constexpr int i = decltype(i_)::value;
                if constexpr (!kDirect && i == kFirst) {
                    k[vPlace].put(lds + kPlace * kTile, wave, lane, S::kSharedKeys);
                    fetch_k(k[vPlace], t + 4, nullptr);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if constexpr (i < kFirst) {
                    constexpr int b = i % kBlocks, x = i / kBlocks;
                    const floatx16 none{};
                    next[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[i % kReads], __builtin_bit_cast(bf16x8, st.qf[x]), x == 0 ? none : next[b], 0, 0, 0);
                } else {
                    constexpr int e = (i - kFirst) / S::kDTiles, d = (i - kFirst) % S::kDTiles;
                    st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[i % kReads], __builtin_bit_cast(bf16x8, pf[e]), st.o[d], 0, 0, 0);
                }
                read(std::integral_constant<int, i + kReads>{});
                if constexpr (i < kFirst) {
                    constexpr int from = i * kEarly / kFirst, to = (i + 1) * kEarly / kFirst;
                    each<to - from>([&](auto n) __attribute__((always_inline)) { pair(std::integral_constant<int, from + decltype(n)::value>{}, s, pf); });
                } else {  // the other pairs, none later than the products before its own, then the maximum
                    constexpr int n = kEarly + i - kFirst, at = i - kFirst - (kPairs - kEarly), kRest = kSecond - (kPairs - kEarly);
                    if constexpr (n < kPairs) pair(std::integral_constant<int, n>{}, s, pf);
                    else
#pragma unroll
                        for (int x = 16 * kBlocks * at / kRest; x < 16 * kBlocks * (at + 1) / kRest; ++x) top = fmaxf(top, next[x / 16][x % 16]);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            if ((t + 2) * S::kSharedKeys > g.shared) {  // (uniform)
                mask_past(next, (t + 1) * S::kSharedKeys, half, g.shared);
                top = largest(next);
            }
            st.rescale(p, top);
        } else if constexpr (!kDirect) {
            k[vPlace].put(lds + kPlace * kTile, wave, lane, S::kSharedKeys);
            fetch_k(k[vPlace], t + 4, nullptr);
        }
        if constexpr (kDirect) {
            if (v_end(t + 1) < S::kSharedKeys) {  // (uniform)
                __builtin_amdgcn_s_waitcnt(0x0070);
                v[0].put(v_to, wave, lane, v_end(t + 1));
            }
            meet<StageK::kLoads>();  // (V of t+1 and K of t+2)
        } else {
            v[vPlace ^ 1].put(v_to, wave, lane, v_end(t + 1), raw + (vPlace ^ 1) * (kTile / 2));
            fetch_v(v[vPlace ^ 1], t + 3, raw + (vPlace ^ 1) * (kTile / 2));
            meet<63>();
        }
    };

    floatx16 even[kBlocks], odd[kBlocks];
    st.sign_q(p);
    if constexpr (kDirect) {
        if (v_end(t0) < S::kSharedKeys) {
            __builtin_amdgcn_s_waitcnt(0x0070);
            v[0].put(lds + kV, wave, lane, v_end(t0));
        }
        meet<StageK::kLoads>();  // (all but the third tile of K)
    } else {
        meet<63>();
    }
    if (active) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int x = 0; x < S::kPieces / 2; ++x) {
                const bf16x8 a = *reinterpret_cast<const bf16x8 *>(lds + (k_at ^ (32 * x)) + b * 32 * S::kRowBytes);
                const floatx16 none{};
                even[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, st.qf[x]), x == 0 ? none : even[b], 0, 0, 0);
            }
        if ((t0 + 1) * S::kSharedKeys > g.shared) mask_past(even, t0 * S::kSharedKeys, half, g.shared);
        st.rescale(p, largest(even));
    }
    meet<kDirect ? StageK::kLoads : 63>();  // (the first tile's K is read by all before it is written over)
    // As many steps in a row as bring both kinds of places around, so that they are constants.
    constexpr int kRound = kRing == 3 ? 6 : 2;
    int t = t0, done = 0;
    for (bool more = t + 1 < t1; more;) {
        each<kRound>([&](auto i_) __attribute__((always_inline)) {
            constexpr int i = decltype(i_)::value;
            if (t + 1 < t1) {
                if constexpr (i % 2 == 0) step(std::integral_constant<int, i % kRing>{}, std::integral_constant<int, i % 2>{}, t, even, odd);
                else step(std::integral_constant<int, i % kRing>{}, std::integral_constant<int, i % 2>{}, t, odd, even);
                ++t;
                done = (i + 1) % 2;
            }
        });
        more = t + 1 < t1;
    }
    if (active) {  // the last tile's exponentials and second product
        if (done == 1)
            for (int b = 0; b < kBlocks; ++b) even[b] = odd[b];
        u32x4 pf[2 * kBlocks];
        each<kPairs>([&](auto n) __attribute__((always_inline)) { pair(n, even, pf); });
#pragma unroll
        for (int i = 0; i < 2 * kBlocks; ++i)
#pragma unroll
            for (int d = 0; d < S::kDTiles; ++d)
                st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v(i, d, done * kTile), __builtin_bit_cast(bf16x8, pf[i]), st.o[d], 0, 0, 0);
    }
    meet<0>();  // (LDS is free)
}

__device__ __attribute__((always_inline)) inline void settle(GroupPlan &g) {  // (every lane has the same: kept in scalar registers)
    for (int32_t *x : {&g.q0, &g.rows, &g.shared, &g.e0, &g.key_tiles, &g.blocks}) *x = __builtin_amdgcn_readfirstlane(*x);
}
// A range of the tiles over shared keys, group after group and block of columns after block: every wave has 32 of the work-group's 128 columns, and the four
// stage the tiles together.
template <Pool POOL, int D>
__device__ __attribute__((always_inline)) inline void shared_work(const SharedParams &p, char *lds, const Job &job) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    int left = job.tiles, tile = job.tile, block = job.block, item = job.item, h = job.outer;
    GroupPlan g = job.g;
    settle(g);
    bool first = true;
    for (;;) {
        const int t1 = min(g.key_tiles, tile + left), last = g.rows * p.G - 1, column0 = block * kBlock + wave * kColumns;
        State<POOL, D> st;
        {
            const int c = min(column0 + col, last), i = by_g(p, c);
            st.clear();
            st.load_q(p, (int64_t)g.q0 + i, h * p.G + c - i * p.G, half);
        }
        shared_tiles(p, lds, g, h, tile, t1, column0 <= last, st);
        const bool whole = tile == 0 && t1 == g.key_tiles;
        if (column0 <= last) {
            int half = lane >> 5, col = lane & 31;
            asm volatile("" : "+v"(half), "+v"(col));  // (as in attend)
            const int packed = column0 + col, i = by_g(p, packed);
            const int64_t to = whole ? ((int64_t)g.q0 + i) * p.Hq + h * p.G + packed - i * p.G : ((int64_t)2 * job.range + !first) * kBlock + wave * kColumns + col;
            write_part(st, sum_of_halves(st.l), either(whole, p.shared_whole_o, p.shared_o), either(whole, p.shared_whole_ml, p.shared_ml), half, packed > last ? -1 : to);
        }
        first = false;
        left -= t1 - tile;
        if (left == 0) break;
        tile = 0;
        if (++block == g.blocks) {
            block = 0;
            do {
                if (++item == p.groups) {
                    item = 0;
                    ++h;
                }
            } while (p.grp[item].key_tiles == 0);
            g = p.grp[item];
            settle(g);
        }
    }
}

// ------------------------------------------------------------------------------------------ keys of a sequence by itself
struct OwnPart {
    int32_t kv_head, packed0, begin_tile, n0, half, col;  // n0: first key of its last tile
    bool whole, final, bad;  // whole: all own keys of the sequence; final: and it shares none; bad: values of V were left out
    int64_t slot;            // of its first column
};

// A wave's columns over the own keys of a sequence, or a part of them: to the output, or to where the parts are joined.
template <Pool POOL, int D>
__device__ __attribute__((always_inline)) inline void own_finish(const SharedParams &p, const State<POOL, D> &st, const SeqPlan &sn, const OwnPart &w) {
    using S = Shape<POOL, D>;
    int half = w.half, col = w.col;
    asm volatile("" : "+v"(half), "+v"(col));  // (as in attend)
    const int lane = half * 32 + col;
    const float l = sum_of_halves(st.l);
    auto row_of = [&](int c) __attribute__((always_inline)) {  // the row and head of column c, as a row of the output
        const int packed = w.packed0 + c, i = by_g(p, packed);
        return packed >= sn.R * p.G ? (int64_t)-1 : ((int64_t)sn.q0 + i) * p.Hq + w.kv_head * p.G + packed - i * p.G;
    };
    char *const part_o = either(w.whole, p.own_whole_o, p.own_o);
    uint32_t wide = 0;
    if (w.final) {
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;  // (no visible key: zero; NaN stays)
        const int64_t mine = row_of(col);
        if (p.lse && half == 0 && mine >= 0) p.lse[mine] = l == 0.f ? -INFINITY : st.m * 0.693147180559945309f + logf(l);
        if constexpr (S::kHalf) {
            write_row<POOL, D, kOutRow>(st, inv, mine < 0 ? nullptr : p.out + mine * S::kRowBytes, half);
        } else if (mine >= 0) {
#pragma unroll
            for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
                for (int x = 0; x < 16; x += 4)
                    *reinterpret_cast<floatx4 *>(p.out + mine * S::kRowBytes + (d * 32 + 2 * x + 4 * half) * 4) =
                        floatx4{st.o[d][x] * inv, st.o[d][x + 1] * inv, st.o[d][x + 2] * inv, st.o[d][x + 3] * inv};
        }
    } else {
        const int64_t at = row_of(col);
        wide = write_part(st, l, part_o, either(w.whole, p.own_whole_ml, p.own_ml), half, at < 0 || w.whole ? at : w.slot + col);
    }
    if (!w.bad) return;
    // The values that put() left out, added to what this wave has written: a column and a d of it per lane.
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    __builtin_amdgcn_wave_barrier();
    // (in the tile that the shared keys end in, and from the first one on that some row does not see all of)
    const int before = sn.L - sn.R, first_key = (sn.shared / 32 + w.begin_tile) * 32, end_key = min(w.n0 + 32, sn.L);
    const int next = first_key < sn.shared ? first_key + 32 : first_key, masked = max(next, max(before, 0) / 32 * 32);
    for (int e = lane; e < kColumns * D; e += 64) {
        const int c = w.packed0 + e / D, d = e % D;
        if (c >= sn.R * p.G) break;
        const int i = by_g(p, c);
        const uint64_t bits = p.tree_mask ? p.tree_mask[sn.q0 + i] : 0;
        float sum = 0.f;
        for (int n = first_key < sn.shared ? sn.shared : masked; n < end_key; n = n + 1 == next ? masked : n + 1) {
            const bool sees = p.tree_mask ? n < before || (n - before < 64 && (bits >> (n - before) & 1)) : n <= before + i;
            if (!sees) continue;
            const int64_t page = max(0, min(p.page_table[sn.e0 + (n >> p.page_shift)], p.num_pages - 1));
            const int slot = n & ((1 << p.page_shift) - 1);
            const int64_t el = (((page << p.page_shift) + slot) * p.Hkv + w.kv_head) * D + d;
            float x;
            if constexpr (POOL == kF32) x = reinterpret_cast<const float *>(p.v)[el];
            else if constexpr (POOL == kBf16) x = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p.v)[el] << 16);
            else {
                uint32_t lo, hi;
                values_of(reinterpret_cast<const uint8_t *>(p.v)[el], scale_of(p.v_scale[((page * p.Hkv + w.kv_head) << p.page_shift) + slot]), lo, hi);
                x = __uint_as_float(lo << 16);
            }
            if (!(fabsf(x) < INFINITY)) sum += x;
        }
        if (sum == 0.f) continue;  // (nothing but infinities and NaN is added)
        const int64_t row = row_of(e / D);
        char *const to = w.final ? p.out + (row * D + d) * S::kSize : part_o + ((w.whole ? row : w.slot + e / D) * D + d) * S::kSize;
        if constexpr (!S::kHalf) *reinterpret_cast<float *>(to) += sum;
        else if (w.final || (wide >> (e / D) & 1)) *reinterpret_cast<__bf16 *>(to) = (__bf16)((float)*reinterpret_cast<__bf16 *>(to) + sum);
        else *reinterpret_cast<_Float16 *>(to) = (_Float16)((float)*reinterpret_cast<_Float16 *>(to) + sum);
    }
}

// A place in the list of own work, and the sequence that it is in.
struct OwnPlace {
    int32_t outer, item, tile;
    SeqPlan s;
    __device__ __attribute__((always_inline)) inline bool next(const SharedParams &p, bool more) {  // whether the tile was its sequence's last; `more`: there is a next one
        if (++tile < s.tiles) return false;
        tile = 0;
        if (more) {
            do {
                if (++item == p.B) {
                    item = 0;
                    ++outer;
                }
            } while (p.seq[item].tiles == 0);
            s = p.seq[item];
        }
        return true;
    }
    __device__ int first_key() const { return (s.shared / 32 + tile) * 32; }
};

// A wave's columns in a sequence, and what each sees of the new tokens.
struct OwnColumns {
    int32_t packed0, begin_tile, lim;
    uint64_t bits;  // (trees)
    template <bool CODES, Pool POOL, int D>
    __device__ __attribute__((always_inline)) inline void begin(const SharedParams &p, const OwnPlace &at, int packed, int kv_head, int half, int col, State<POOL, D> &st) {
        packed0 = packed;
        begin_tile = at.tile;
        const int last = at.s.R * p.G - 1, c = min(packed0 + col, last), i = by_g(p, c);
        lim = at.s.L - at.s.R + i + 1;
        if (p.tree_mask) bits = p.tree_mask[at.s.q0 + i];
        st.clear();
        st.template load_q<CODES>(p, (int64_t)at.s.q0 + i, kv_head * p.G + c - i * p.G, half);
    }
    // Score x of a tile is key n0 + 8 (x / 4) + 4 half + x % 4.
    __device__ __attribute__((always_inline)) inline void mask(const SharedParams &p, const SeqPlan &s, int n0, int half, floatx16 &sc) const {
        const int before = s.L - s.R;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const int n = n0 + 8 * (x / 4) + 4 * half + x % 4;
            const bool sees = p.tree_mask ? n < before || (n < s.L && n - before < 64 && (bits >> (n - before) & 1)) : n < lim;
            if (n < s.shared || !sees) sc[x] = -INFINITY;
        }
    }
};

// 8 bits: K and V of two tiles at a time are on their way into a wave's part of LDS as they are, each lane asking for the piece that belongs where its sixteen
// bytes land.  They are turned into bf16 behind the reads that the products take them by: sixteen codes of a key's K, and by the transposing read of bytes
// (sixteen lanes address eight keys by sixteen d and receive one d of the eight keys each) eight of V, whose scales go to the probabilities.  So neither
// the registers nor LDS hold a tile twice (those trees: 178 us by registers and bf16 in LDS, 173 so).  bf16 goes through registers: straight into LDS there is
// room for one tile to a wave only, which is asked for after the one before it has been read (32 groups of 8, 28/4 heads: 191 us, 184 by registers).
template <int D>
struct Codes {
    using S = Shape<kE4m3, D>;
    static constexpr int kLoads = S::kOwnLoads, kRun = 16 / S::kLoadKeys;
    static __device__ int place(int key, int piece) { return D == 128 ? piece ^ ((key >> 1) & 7) : piece ^ ((key >> 2) & 3); }  // (its own inverse)
    template <bool V>
    static __device__ __attribute__((always_inline)) inline void load(const SharedParams &p, const Runs &runs, int h, int lane, char *to) {
        const uint32_t token = (uint32_t)p.Hkv * D;
#pragma unroll
        for (int run = 0; run < kLoads / kRun; ++run) {
            const Run &r = runs[run];
            const char *from = (V ? p.v : p.k) + r.row(p, h) * D;
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                const int in_run = j * S::kLoadKeys + lane / S::kPoolPieces;
                const uint32_t off = (uint32_t)min(in_run, r.left) * token + (uint32_t)place(run * 16 + in_run, lane % S::kPoolPieces) * 16;
                __builtin_amdgcn_global_load_lds((GlobalFrom)(from + off), (LdsTo)(to + (run * kRun + j) * 1024), 16, 0, 2);  // (past the caches: read once)
            }
        }
    }
    // The scale bytes of K of key `lane`, of V of key `lane` - 32.
    static __device__ __attribute__((always_inline)) inline uint32_t load_scale(const SharedParams &p, const Runs &r, int h, int lane) {
        const int key = lane & 31;
        const int64_t at = key < 16 ? r.a.scale(p, h) + min(key, r.a.left) : r.b.scale(p, h) + min(key - 16, r.b.left);
        return (lane < 32 ? p.k_scale : p.v_scale)[at];
    }
};

// Sixteen bytes of V in LDS where some row does not see all keys: what is not finite counts as zero (it is added at the end to the rows that see it), as does all
// of a key that is no row's (`none`).  Whether there was something not finite.
template <bool CODES>
__device__ inline bool sift(char *at, bool none) {
    u32x4 x = *reinterpret_cast<const u32x4 *>(at);
    bool bad = false;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        // (codes: a one for each byte that is 0x7f or 0xff)
        const uint32_t nan = CODES ? ((((x[w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu
                                   : ((x[w] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u) | ((x[w] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u);
        bad |= nan != 0 && !none;
        x[w] &= none ? 0u : ~nan;
    }
    *reinterpret_cast<u32x4 *>(at) = x;
    return bad;
}

__device__ inline bf16x8 eight_of(uint32_t lo, uint32_t hi, float scale) {
    u32x4 y;
    uint32_t a, b;
    values_of(lo, scale, a, b);
    y[0] = a;
    y[1] = b;
    values_of(hi, scale, a, b);
    y[2] = a;
    y[3] = b;
    return __builtin_bit_cast(bf16x8, y);
}
__device__ inline void lds_read() {  // what the wave has asked LDS for is there
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
}
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef i32x2 __attribute__((address_space(3))) *LdsTrBytes;

// A tile of 32 keys as codes (K at `k` of `lds`, V at `v`; `scales` of K's keys, then of V's) into the state; between() once they have been read.
template <int D, typename Between, typename Mask>
__device__ __attribute__((always_inline)) inline void attend_codes(const SharedParams &p, State<kE4m3, D> &st, char *lds, int k, int v, const float *scales, bool active,
                                                                   int half, int col, Between &&between, Mask &&mask) {
    using S = Shape<kE4m3, D>;
    typedef Codes<D> C;
    const int lane = half * 32 + col;
    // Where this lane reads: a key's K; of V, the row of its pair of lanes, eight bytes of the sixteen that its group receives.
    const int v_key = 8 * ((lane & 15) >> 3) + 4 * half + ((lane & 15) >> 1) % 4;
    int k_at = k + col * D + C::place(col, half) * 16, v_at = v + v_key * D + (lane & 1) * 8;
    asm volatile("" : "+v"(k_at), "+v"(v_at));
    // All of the tile's codes into registers, so that its place is free for the tile that between() asks for (256 sequences of 512 to 4,096 tokens at 28/4 heads: 128 us
    // with V read and asked for after the scores, 116 so).
    u32x4 kc[D / 32];
    i32x2 vc[2][S::kDTiles];
    floatx4 v_scale[4];
    float k_scale;
    if (active) {
#pragma unroll
        for (int y = 0; y < D / 32; ++y) kc[y] = *reinterpret_cast<const u32x4 *>(lds + (k_at ^ (32 * y)));
        k_scale = scales[col];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int d = 0; d < S::kDTiles; ++d)
                vc[i][d] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((LdsTrBytes)(lds + v_at + i * 16 * D + C::place(i * 16 + v_key, 2 * d + ((lane >> 4) & 1)) * 16));
#pragma unroll
        for (int i = 0; i < 4; ++i) v_scale[i] = *reinterpret_cast<const floatx4 *>(scales + 32 + 8 * i + 4 * half);
    }
    between();
    if (!active) return;
    floatx16 s, other;
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = other[x] = 0.f;
#pragma unroll
    for (int y = 0; y < D / 32; ++y) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(eight_of(kc[y][0], kc[y][1], k_scale), __builtin_bit_cast(bf16x8, st.qf[2 * y]), s, 0, 0, 0);
        other = __builtin_amdgcn_mfma_f32_32x32x16_bf16(eight_of(kc[y][2], kc[y][3], k_scale), __builtin_bit_cast(bf16x8, st.qf[2 * y + 1]), other, 0, 0, 0);
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] += other[x];
    mask(s);
    st.exponentials(p, s);
    u32x4 pf[2];
#pragma unroll
    for (int i = 0; i < 4; ++i)  // (a power of two: nothing but the exponent moves)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            pf[i / 2][i % 2 * 2 + j] = __builtin_bit_cast(
                uint32_t, __builtin_convertvector(floatx2{s[4 * i + 2 * j] * v_scale[i][2 * j], s[4 * i + 2 * j + 1] * v_scale[i][2 * j + 1]}, bf16x2));
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
            st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(eight_of((uint32_t)vc[i][d][0], (uint32_t)vc[i][d][1], 1.f), __builtin_bit_cast(bf16x8, pf[i]), st.o[d], 0, 0, 0);
}

// Every wave walks a range of its own, without barriers, in tiles of 32 keys.  Neighbouring waves have neighbouring KV heads of the same keys.
template <Pool POOL, int D>
__device__ __attribute__((always_inline)) inline void own_work(const SharedParams &p, char *lds, const Job &job) {
    using S = Shape<POOL, D>;
    constexpr bool kCodes = POOL == kE4m3;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    const int cw = wave % p.col_waves, hi = wave / p.col_waves % p.heads_wg, n_tiles = job.tiles;
    const int head_groups = p.Hkv / p.heads_wg;
    const int at0 = wave * S::kOwnBytes;  // of the wave's part of LDS
    char *const mine = lds + at0;
    OwnPlace now{job.outer, job.item, job.tile, job.s}, ahead = now;
    State<POOL, D> st;
    OwnColumns cols{};
    bool fresh = true, first = true, bad = false;
    auto head_of = [&](const OwnPlace &x) __attribute__((always_inline)) { return x.outer % head_groups * p.heads_wg + hi; };
    auto look = [&]() __attribute__((always_inline)) { return Runs(p, ahead.s.e0, ahead.first_key(), ahead.s.L - 1); };
    Runs runs = look();  // of the next tile to fetch
    auto begin = [&]() __attribute__((always_inline)) {
        cols.template begin<kCodes>(p, now, (now.outer / head_groups * p.col_waves + cw) * kColumns, head_of(now), half, col, st);
    };
    auto finish = [&](const SeqPlan &sn, int tile, int n0, int kv_head) __attribute__((always_inline)) {  // after the sequence's or the range's last tile
        const bool whole = cols.begin_tile == 0 && tile + 1 == sn.tiles;
        if (cols.packed0 < sn.R * p.G)
            own_finish<POOL, D>(p, st, sn, OwnPart{kv_head, cols.packed0, cols.begin_tile, n0, half, col, whole, whole && sn.shared == 0, __ballot(bad) != 0,
                                                   (((int64_t)2 * job.range + !first) * (4 / p.parts_wg) + hi * p.col_waves + cw) * kColumns});
        bad = first = false;
    };
    if constexpr (!kCodes) {
        char *const kt = mine, *const vt = mine + S::kOwnBytes / 2;
        Mover<POOL, D> mover;
        auto fetch = [&](int f) __attribute__((always_inline)) {  // the tile that is f-th of this range, on its way while the one before it is read
            mover.load(p, runs, head_of(ahead), lane);
            ahead.next(p, f + 1 < n_tiles);
            runs = look();
        };
        fetch(0);
        for (int f = 0; f < n_tiles; ++f) {
            const SeqPlan sn = now.s;
            const int tile = now.tile, kv_head = head_of(now), n0 = now.first_key();
            const bool special = n0 < sn.shared || n0 + 32 > sn.L - sn.R + (p.tree_mask ? 0 : 1);  // some row does not see all of its keys
            if (fresh) begin();
            if (special) bad |= mover.template put<true>(kt, vt, lane, n0, sn.shared, sn.L);
            else mover.template put<false>(kt, vt, lane, 0, 0, 0);
            if (fresh) st.sign_q(p);
            if (f + 1 < n_tiles) fetch(f + 1);
            fresh = now.next(p, f + 1 < n_tiles);
            wave_sync();
            if (cols.packed0 < sn.R * p.G)  // (uniform)
                attend(p, st, lds, at0, at0 + S::kOwnBytes / 2, half, col, [&](floatx16 &sc) __attribute__((always_inline)) {
                    if (special) cols.mask(p, sn, n0, half, sc);
                });
            wave_sync();
            if (fresh || f + 1 == n_tiles) finish(sn, tile, n0, kv_head);
        }
    } else {
        typedef Codes<D> C;
        float *const scales = reinterpret_cast<float *>(mine + 4 * S::kCodeBytes);  // of K of the tile's keys, and of V
        uint32_t sc_byte[2] = {0, 0};
        auto fetch = [&](int f, uint32_t &byte) __attribute__((always_inline)) {  // (the scales last: a step goes by them)
            C::template load<false>(p, runs, head_of(ahead), lane, mine + f % 2 * S::kCodeBytes);
            C::template load<true>(p, runs, head_of(ahead), lane, mine + (2 + f % 2) * S::kCodeBytes);
            asm volatile("" ::: "memory");
            byte = C::load_scale(p, runs, head_of(ahead), lane);
            ahead.next(p, f + 1 < n_tiles);
            runs = look();
        };
        begin();
        fetch(0, sc_byte[0]);
        if (1 < n_tiles) fetch(1, sc_byte[1]);
        auto step = [&](auto place_, int f) __attribute__((always_inline)) {
            constexpr int kPlace = decltype(place_)::value;
            const SeqPlan sn = now.s;
            const int tile = now.tile, kv_head = head_of(now), n0 = now.first_key();
            const bool special = n0 < sn.shared || n0 + 32 > sn.L - sn.R + (p.tree_mask ? 0 : 1);
            if (fresh && f > 0) begin();
            asm volatile("" ::"v"(sc_byte[kPlace]) : "memory");  // (loads come back in order: the tile is there)
            char *const vt = mine + (2 + kPlace) * S::kCodeBytes;
            float scale = scale_of((int)sc_byte[kPlace]);
            if (special) {
                for (int i = 0; i < S::kOwnLoads; ++i) {
                    const int n = n0 + i * S::kLoadKeys + lane / S::kPoolPieces;
                    bad |= sift<true>(vt + i * 1024 + lane * 16, n < sn.shared || n >= sn.L);
                }
                if (lane >= 32 && (n0 + lane - 32 < sn.shared || n0 + lane - 32 >= sn.L)) scale = 0.f;
            }
            scales[lane] = scale;
            if (fresh) st.sign_q(p);
            fresh = now.next(p, f + 1 < n_tiles);
            wave_sync();
            const bool active = cols.packed0 < sn.R * p.G;
            attend_codes<D>(p, st, mine, kPlace * S::kCodeBytes, (2 + kPlace) * S::kCodeBytes, scales, active, half, col,
                            [&]() __attribute__((always_inline)) {
                                if (f + 2 < n_tiles) {
                                    lds_read();  // (before its place is written over)
                                    fetch(f + 2, sc_byte[kPlace]);
                                }
                            },
                            [&](floatx16 &sc) __attribute__((always_inline)) {
                                if (special) cols.mask(p, sn, n0, half, sc);
                            });
            if (fresh || f + 1 == n_tiles) finish(sn, tile, n0, kv_head);
        };
        for (int f = 0; f < n_tiles; f += 2) {
            step(std::integral_constant<int, 0>{}, f);
            if (f + 1 < n_tiles) step(std::integral_constant<int, 1>{}, f + 1);
        }
    }
}

// 8 bits, more than 32 columns to a KV head: CW waves with 32 of them each walk one range together and share its tiles, which lie in LDS as they do in the pool.
// All of the work-group's waves, on 4 / CW heads, go from tile to tile at the same time: a step begins with a barrier, then asks for the tile three further on,
// in the place of the one that was read in the step before.  (A tile that each wave loads for itself is asked for CW times, and a compute unit can only
// have so much on its way: those trees 158 us, 142 so.  bf16 tiles are twice as large, the code for them beside this cost the shared keys 5 %.)
template <int D, int CW>
__device__ __attribute__((always_inline)) inline void paired_work(const SharedParams &p, char *lds, const Job &job) {
    using S = Shape<kE4m3, D>;
    constexpr int kRing = S::kPairedRing, kHeads = 4 / CW, kLoads = 2 * S::kOwnLoads / CW, kGroup = kLoads + 1, kRun = 16 / S::kLoadKeys;  // (of K and V, of a wave)
    static_assert(kHeads <= S::kPairedHeads && kLoads >= 1, "the tiles fit");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31, cw = wave % CW, hi = wave / CW, n_tiles = job.tiles, head_groups = p.Hkv / kHeads;
    char *const ring = lds + hi * kRing * S::kTileBytes;
    char *const bytes = lds + kHeads * kRing * S::kTileBytes + hi * kRing * 64;                                // scales of K and V of each tile
    int *const flags = reinterpret_cast<int *>(lds + kHeads * kRing * (S::kTileBytes + 64)) + hi * kRing;       // whether V of a tile held something not finite
    float *const scales = reinterpret_cast<float *>(lds + kHeads * kRing * (S::kTileBytes + 64 + 16)) + wave * 2 * S::kOwnKeys;
    OwnPlace now{job.outer, job.item, job.tile, job.s}, ahead = now;
    State<kE4m3, D> st;
    OwnColumns cols{};
    bool fresh = true, first = true, bad = false;
    auto head_of = [&](const OwnPlace &x) __attribute__((always_inline)) { return x.outer % head_groups * kHeads + hi; };
    auto look = [&]() __attribute__((always_inline)) { return Runs(p, ahead.s.e0, ahead.first_key(), ahead.s.L - 1); };
    Runs r = look();  // of the next tile to fetch
    auto begin = [&]() __attribute__((always_inline)) {
        cols.template begin<true>(p, now, (now.outer / head_groups * CW + cw) * kColumns, head_of(now), half, col, st);
    };
    // Load i of a tile's is its wave's i / CW-th, for K and then for V; keys run * 16 + j * kLoadKeys on.
    auto fetch = [&](int f) __attribute__((always_inline)) {
        const int h = head_of(ahead);
        char *const to = ring + f % kRing * S::kTileBytes;
        const uint32_t token = (uint32_t)p.Hkv * D;
#pragma unroll
        for (int y = 0; y < kLoads; ++y) {
            const int i = y * CW + cw, at = i % S::kOwnLoads, run = at / kRun, in_run = at % kRun * S::kLoadKeys + lane / S::kPoolPieces, key = run * 16 + in_run;
            const char *from = (i >= S::kOwnLoads ? p.v : p.k) + (run == 0 ? r[0].row(p, h) : r[1].row(p, h)) * D;
            const uint32_t off = (uint32_t)min(in_run, run == 0 ? r[0].left : r[1].left) * token + (uint32_t)Codes<D>::place(key, lane % S::kPoolPieces) * 16;
            __builtin_amdgcn_global_load_lds((GlobalFrom)(from + off), (LdsTo)(to + i * 1024), 16, 0, 2);
        }
        // sixteen lanes with four scales each: K's of both runs, V's of both (those past the last key are not used)
        if (lane < 16) {
            const int64_t at = (lane & 4 ? r[1].scale(p, h) - (r[1].slot & 15) : r[0].scale(p, h) - (r[0].slot & 15)) + (lane & 3) * 4;
            __builtin_amdgcn_global_load_lds((GlobalFrom)((lane & 8 ? p.v_scale : p.k_scale) + at), (LdsTo)(bytes + f % kRing * 64), 4, 0, 0);
        }
        ahead.next(p, f + 1 < n_tiles);
        r = look();
    };
    if (lane < kRing && cw == 0) flags[lane] = 0;
    fetch(0);
    begin();
    if (1 < n_tiles) fetch(1);
    if (2 < n_tiles) fetch(2);
    meet<63>();
    for (int f = 0; f < n_tiles; ++f) {
        const SeqPlan sn = now.s;
        const int tile = now.tile, kv_head = head_of(now), n0 = now.first_key(), place = f % kRing;
        const bool special = n0 < sn.shared || n0 + 32 > sn.L - sn.R + (p.tree_mask ? 0 : 1);  // some row does not see all of its keys
        char *const here = ring + place * S::kTileBytes;
        // This wave's loads of the tile are there, those of the next two may not be.
        if (f + 2 < n_tiles) wait_for<2 * kGroup>();
        else if (f + 1 < n_tiles) wait_for<kGroup>();
        else wait_for<0>();
        if (special) {
            bool mine = false;
#pragma unroll
            for (int y = 0; y < kLoads; ++y) {
                const int i = y * CW + cw, key = (i % S::kOwnLoads) * S::kLoadKeys + lane / S::kPoolPieces;
                if (i >= S::kOwnLoads) mine |= sift<true>(here + i * 1024 + lane * 16, n0 + key < sn.shared || n0 + key >= sn.L);
            }
            if (mine) flags[place] = 1;
        }
        meet<63>();  // (the tile is there, and the one before has been read)
        if (fresh && f > 0) begin();
        if (f + 3 < n_tiles) fetch(f + 3);
        if (special) bad |= flags[place] != 0;
        if (cw == 0 && lane == 0) flags[(f + 2) % kRing] = 0;
        const bool active = cols.packed0 < sn.R * p.G;  // (uniform)
        if (fresh) st.sign_q(p);
        fresh = now.next(p, f + 1 < n_tiles);
        float scale = scale_of((int)reinterpret_cast<const uint8_t *>(bytes)[place * 64 + lane]);
        if (special && lane >= 32 && (n0 + lane - 32 < sn.shared || n0 + lane - 32 >= sn.L)) scale = 0.f;
        scales[lane] = scale;
        wave_sync();
        attend_codes<D>(p, st, here, 0, S::kTileBytes / 2, scales, active, half, col, []() {}, [&](floatx16 &sc) __attribute__((always_inline)) {
            if (special) cols.mask(p, sn, n0, half, sc);
        });
        wave_sync();
        if (!fresh && f + 1 < n_tiles) continue;
        const bool whole = cols.begin_tile == 0 && tile + 1 == sn.tiles;
        if (active)
            own_finish<kE4m3, D>(p, st, sn, OwnPart{kv_head, cols.packed0, cols.begin_tile, n0, half, col, whole, whole && sn.shared == 0, __ballot(bad) != 0,
                                                   (((int64_t)2 * job.range + !first) * 4 + hi * CW + cw) * kColumns});
        bad = first = false;
    }
}

template <Pool POOL, int D>
__global__ __launch_bounds__(kThreads, POOL == kF32 ? 1 : 2) void shared_attention_kernel(SharedParams p) {
    extern __shared__ __align__(16) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Job &job = p.jobs[blockIdx.x * 4 + wave / (4 / p.parts_wg)];
    if (job.key != p.key) return;  // (no plan of these sizes)
    if (job.kind == kShared) shared_work<POOL, D>(p, lds, job);
    else if (job.kind == kOwn) {
        if constexpr (POOL == kE4m3) {
            if (p.col_waves == 4) return paired_work<D, 4>(p, lds, job);
            if (p.col_waves == 2) return paired_work<D, 2>(p, lds, job);
        }
        own_work<POOL, D>(p, lds, job);
    }
}

// ------------------------------------------------------------------------------------------ joining the parts
// D / 8 lanes for each row and head of a sequence; SPLIT: in each of the work-group's waves, which share the parts out and add up through LDS what they found.
// Each lane looks at the maximum and sum of another part; the outputs are then weighted and summed in the parts' order, those of shared keys first, without
// one load waiting for another.
template <bool HALF, int D, bool SPLIT>
__global__ __launch_bounds__(kThreads) void shared_join_kernel(SharedParams p) {
    constexpr int kLanes = D / 8, kWaves = kThreads / 64, kPer = (SPLIT ? 64 : kThreads) / kLanes;
    __shared__ float lds[SPLIT ? kWaves * kPer * (D + 4) : 1];
    const Totals t = *p.totals;
    const SeqPlan s = p.seq[blockIdx.y];
    SeqGroup g{};
    if (p.groups > 0) g = p.seq_grp[blockIdx.y];  // (of no meaning where the sequence shares nothing)
    const int wave = threadIdx.x >> 6, part = threadIdx.x % kLanes, sub = (SPLIT ? threadIdx.x & 63 : threadIdx.x) / kLanes;
    const int last = s.R * p.Hq - 1, item = min((int)blockIdx.x * kPer + sub, last);
    if (t.key != p.key || (int)blockIdx.x * kPer > last) return;
    const bool exists = (int)blockIdx.x * kPer + sub <= last;
    const int i = item / p.Hq, head = item - i * p.Hq, kv_head = head / p.G, g_head = head - kv_head * p.G, c = i * p.G + g_head;
    const int64_t row = s.q0 + i, at = row * p.Hq + head;
    int n_shared = 0, n_own = 0;
    // Where the parts of each kind lie, in rows of D (and of their four words): the first one, and how far apart they are.
    const char *shared_o = p.shared_whole_o, *own_o = p.own_whole_o;
    const float *shared_ml = p.shared_whole_ml, *own_ml = p.own_whole_ml;
    int64_t shared_at = at, own_at = at;
    int shared_late = 0, own_late = 0;  // rows further where the first part is its range's last one, not its first
    constexpr int kSharedStep = 2 * kBlock;
    const int own_step = 2 * p.heads_wg * p.col_waves * kColumns;
    if (s.shared > 0) {
        const int packed = max(0, min((int)(row - g.q0) * p.G + g_head, g.rows * p.G - 1));
        const int64_t b = t.shared_step * kv_head + g.base + (int64_t)(packed / kBlock) * (g.key_tiles + t.shared_head);
        const int r = range_of(t.shared, b + t.shared_head);
        n_shared = range_of(t.shared, b + t.shared_head + g.key_tiles - 1) - r + 1;
        if (n_shared > 1) {
            shared_o = p.shared_o;
            shared_ml = p.shared_ml;
            shared_at = (int64_t)r * kSharedStep + packed % kBlock;
            shared_late = begin_of(t.shared, r) < b ? kSharedStep / 2 : 0;
        }
    }
    if (s.tiles > 0) {
        const int cols = p.col_waves * kColumns, c_block = c / cols, c_in = c - c_block * cols, head_block = kv_head / p.heads_wg;
        const int64_t b = t.own_step * (c_block * (p.Hkv / p.heads_wg) + head_block) + s.base;
        const int r = range_of(t.own, b + t.own_head);
        n_own = range_of(t.own, b + t.own_head + s.tiles - 1) - r + 1;
        if (n_own > 1) {
            own_o = p.own_o;
            own_ml = p.own_ml;
            own_at = (int64_t)r * own_step + (kv_head - head_block * p.heads_wg) * cols + c_in;
            own_late = begin_of(t.own, r) < b ? own_step / 2 : 0;
        }
    }
    const bool written = n_own == 1 && n_shared == 0;  // (already)
    float m = -INFINITY, l = 0.f;
    float o[8] = {};
    constexpr int kRowBytes = D * (HALF ? 2 : 4);
    const int n = written ? 0 : n_shared + n_own, share = SPLIT ? (n + kWaves - 1) / kWaves : n;
    const int begin = SPLIT ? min(n, wave * share) : 0, end = SPLIT ? min(n, begin + share) : n;
    constexpr int kWords = HALF ? 1 : 2;
    // N parts at a time, all asked for before the first is waited for (one behind the other they take 0.8 us each).
    auto ask = [&](int j, int to, auto &x) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(x) / sizeof(x[0])); ++i) {
            const int at_part = min(j + i, to - 1), in_own = at_part - n_shared;
            const char *from = in_own < 0 ? shared_o + (shared_at + (int64_t)at_part * kSharedStep + (at_part == 0 ? shared_late : 0)) * kRowBytes
                                          : own_o + (own_at + (int64_t)in_own * own_step + (in_own == 0 ? own_late : 0)) * kRowBytes;
#pragma unroll
            for (int y = 0; y < kWords; ++y) x[i][y] = *reinterpret_cast<const u32x4 *>(from + part * (HALF ? 16 : 32) + 16 * y);
        }
    };
    for (int j0 = begin; j0 < end; j0 += kLanes) {
        const int mine = j0 + part, in_own = mine - n_shared, to = min(end, j0 + kLanes), lane0 = (int)(threadIdx.x & 63) / kLanes * kLanes;
        floatx4 ml = {-INFINITY, 0.f, 0.f, 0.f};
        if (mine < end)
            ml = in_own < 0 ? reinterpret_cast<const floatx4 *>(shared_ml)[shared_at + (int64_t)mine * kSharedStep + (mine == 0 ? shared_late : 0)]
                            : reinterpret_cast<const floatx4 *>(own_ml)[own_at + (int64_t)in_own * own_step + (in_own == 0 ? own_late : 0)];
        float e = 0.f;
        bool any_wide = false;  // of these parts
        auto weigh = [&]() __attribute__((always_inline)) {
            if (ml[1] == 0.f) ml[0] = -INFINITY;  // (no key of this part is seen)
            float top = ml[0];
#pragma unroll
            for (int step = 1; step < kLanes; step *= 2) top = fmaxf(top, __shfl_xor(top, step));
            const float m_new = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
            e = ml[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[0] - m_new);
            float sum = ml[1] * e;
            e *= ml[2];  // (of the output, in its unit; negative for a wide row)
            if constexpr (HALF) {
                any_wide = __ballot(ml[3] != 0.f) != 0;
                if (ml[3] != 0.f) e = -e;
            }
#pragma unroll
            for (int step = 1; step < kLanes; step *= 2) sum += __shfl_xor(sum, step);
            l = l * f + sum;
            for (int x = 0; x < 8; ++x) o[x] *= f;
            m = m_new;
        };
        auto sum_up = [&](int j, auto &x, auto wide_) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < (int)(sizeof(x) / sizeof(x[0])); ++i) {
                const float w = __shfl(e, lane0 + min(j + i, to - 1) - j0);
                if (j + i >= to)
#pragma unroll
                    for (int y = 0; y < kWords; ++y) x[i][y] = u32x4{0, 0, 0, 0};
                if constexpr (HALF) {
                    const halfx8 h = __builtin_bit_cast(halfx8, x[i][0]);
                    if constexpr (!decltype(wide_)::value) {
                        for (int y = 0; y < 8; ++y) o[y] = fmaf((float)h[y], w, o[y]);
                    } else {
                        for (int y = 0; y < 8; ++y) {
                            const uint32_t word = x[i][0][y / 2];
                            o[y] = fmaf(__float_as_int(w) < 0 ? __uint_as_float(y % 2 ? word & 0xffff0000u : word << 16) : (float)h[y], fabsf(w), o[y]);
                        }
                    }
                } else {
                    const floatx4 a = __builtin_bit_cast(floatx4, x[i][0]), b = __builtin_bit_cast(floatx4, x[i][kWords - 1]);
                    for (int y = 0; y < 8; ++y) o[y] = fmaf(y < 4 ? a[y % 4] : b[y % 4], w, o[y]);
                }
            }
        };
        auto add = [&](int j, auto &x) __attribute__((always_inline)) {
            if (any_wide) sum_up(j, x, std::true_type{});
            else sum_up(j, x, std::false_type{});
        };
        if (__ballot(to - j0 > 2) == 0) {  // (most sequences of a large batch)
            u32x4 x[2][kWords];
            ask(j0, to, x);
            weigh();
            add(j0, x);
        } else {
            u32x4 x[HALF ? 8 : 4][kWords];
            ask(j0, to, x);
            weigh();
            add(j0, x);
            for (int j = j0 + (HALF ? 8 : 4); j < to; j += HALF ? 8 : 4) {
                ask(j, to, x);
                add(j, x);
            }
        }
    }
    if constexpr (SPLIT) {
        float *const mine = lds + (wave * kPer + sub) * (D + 4);
        for (int y = 0; y < 8; ++y) mine[y * kLanes + part] = o[y];
        if (part == 0) *reinterpret_cast<floatx2 *>(mine + D) = floatx2{m, l};
        __syncthreads();
        if (wave != 0) return;
        for (int w = 1; w < kWaves; ++w) {
            const float *other = lds + (w * kPer + sub) * (D + 4);
            const floatx2 ml = *reinterpret_cast<const floatx2 *>(other + D);
            const float m_new = fmaxf(m, ml[0]);
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new), e = ml[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[0] - m_new);
            l = l * f + ml[1] * e;
            for (int y = 0; y < 8; ++y) o[y] = o[y] * f + other[y * kLanes + part] * e;
            m = m_new;
        }
    }
    if (written || !exists) return;
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    for (int j = 0; j < 8; ++j) o[j] *= inv;
    if constexpr (HALF) {
        u32x4 y;
        for (int j = 0; j < 4; ++j) y[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{o[2 * j], o[2 * j + 1]}, bf16x2));
        __builtin_nontemporal_store(y, reinterpret_cast<u32x4 *>(p.out + at * kRowBytes + part * 16));
    } else {
        *reinterpret_cast<floatx4 *>(p.out + at * kRowBytes + part * 32) = floatx4{o[0], o[1], o[2], o[3]};
        *reinterpret_cast<floatx4 *>(p.out + at * kRowBytes + part * 32 + 16) = floatx4{o[4], o[5], o[6], o[7]};
    }
    if (p.lse && part == 0) p.lse[at] = l == 0.f ? -INFINITY : m * 0.693147180559945309f + logf(l);
}

// ------------------------------------------------------------------------------------------ host side
// The workspace, piece by piece, each at a multiple of 256 bytes.
struct Layout {
    size_t seq, seq_grp, grp, jobs, totals, own_o, own_ml, shared_o, shared_ml, own_whole_o, own_whole_ml, shared_whole_o, shared_whole_ml, bytes;
};
Layout layout(int32_t B, int32_t total_q, int32_t groups, int32_t Hq, int32_t D, respec_dtype_t dt) {
    Layout w{};
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t here = at;
        at += round_up(n, 256);
        return here;
    };
    const size_t ml = 4 * sizeof(float), o = (size_t)D * (dt == RESPEC_BF16 ? 2 : 4);
    const size_t rows = groups > 0 ? (size_t)total_q * Hq : 0, own = (size_t)kWorkGroups * 8 * kColumns, shared = groups > 0 ? (size_t)kWorkGroups * 2 * kBlock : 0;
    w.seq = take((size_t)B * sizeof(SeqPlan));
    w.seq_grp = take(groups > 0 ? (size_t)B * sizeof(SeqGroup) : 0);
    w.grp = take((size_t)groups * sizeof(GroupPlan));
    w.jobs = take(kJobs * sizeof(Job));
    w.totals = take(sizeof(Totals));
    w.own_ml = take(own * ml);
    w.own_o = take(own * o);
    w.shared_ml = take(shared * ml);
    w.shared_o = take(shared * o);
    w.own_whole_ml = take(rows * ml);
    w.own_whole_o = take(rows * o);
    w.shared_whole_ml = take(rows * ml);
    w.shared_whole_o = take(rows * o);
    w.bytes = at;
    return w;
}

bool sizes_fit(int32_t B, int32_t total_q, int32_t groups, int32_t max_q, int32_t max_kv, int32_t Hq, int32_t Hkv, int32_t D, respec_dtype_t dt) {
    if (B <= 0 || total_q <= 0 || groups < 0 || max_q <= 0 || max_kv <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0) return false;
    if ((D != 64 && D != 128) || (dt != RESPEC_F32 && dt != RESPEC_BF16)) return false;
    return (int64_t)(Hq / Hkv) * max_q <= 256 && (int64_t)total_q * Hq < (1 << 30) && max_kv <= INT32_MAX - 256;
}

template <Pool POOL, int D>
hipError_t launch(const SharedParams &p, bool prepared, hipStream_t stream) {
    using S = Shape<POOL, D>;
    // (in LDS by eight work-groups 1,024 sequences take 11.5 us, 14.4 in 128 groups; in memory by one work-group 1,025 take 21, 4,096 41, 79 in 512 groups)
    if (!prepared && p.B <= kFewSeqs && p.groups <= kFewGroups)
        hipLaunchKernelGGL((shared_prep_kernel<S::kSharedKeys, true>), dim3(kPrepGroups), dim3(kPrepThreads), 0, stream, p);
    else if (!prepared)
        hipLaunchKernelGGL((shared_prep_kernel<S::kSharedKeys, false>), dim3(1), dim3(kPrepThreads), 0, stream, p);
    auto *kernel = &shared_attention_kernel<POOL, D>;
    if (S::kLdsBytes > 65536) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::kLdsBytes);
        if (err != hipSuccess) return err;
    }
    mark_before_main(stream);
    hipLaunchKernelGGL(kernel, dim3(kWorkGroups), dim3(kThreads), S::kLdsBytes, stream, p);
    mark_after_main(stream);
    // Few rows have many parts each, which four waves share out: single tokens over 8 bits at 28/4 heads, a call with and without, 448 rows and heads 23.9 and 30.2 us,
    // 1,792 36.3 and 37.3, 3,584 58.8 and 57.0, 7,168 101.7 and 97.1; groups in bf16 21.8 and 24.7, 29.6 and 31.0, 39.3 and 37.3, 63.2 and 58.5.
    const bool split = (int64_t)p.total_q * p.Hq <= 4096;
    const int per = (split ? 64 : kThreads) / (D / 8);
    const dim3 grid((unsigned)((p.max_q * p.Hq + per - 1) / per), (unsigned)p.B);
    if (split) hipLaunchKernelGGL((shared_join_kernel<S::kHalf, D, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((shared_join_kernel<S::kHalf, D, false>), grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}

respec_status_t run(const char *name, SharedParams &p, int32_t D, int32_t page_size, float sm_scale, respec_dtype_t dt, respec_dtype_t pool_dt, bool prepared,
                    void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!p.q || !p.k || !p.v || !p.q_indptr || !p.page_indptr || !p.page_table || !p.kv_len || !p.out) return fail(RESPEC_ERR_INVALID_ARG, "%s: null pointer argument", name);
    if (p.groups < 0 || (p.groups > 0 && (!p.group_indptr || !p.shared_len))) return fail(RESPEC_ERR_INVALID_ARG, "%s: groups without group_indptr or shared_len", name);
    if (p.B <= 0 || p.total_q <= 0 || p.num_pages <= 0 || p.table_len <= 0 || p.max_q <= 0 || p.max_kv <= 0 || p.Hq <= 0 || p.Hkv <= 0)
        return fail(RESPEC_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d total_q=%d max_q=%d max_kv=%d Hq=%d Hkv=%d)", name, p.B, p.total_q, p.max_q, p.max_kv, p.Hq, p.Hkv);
    if (p.Hq % p.Hkv != 0) return fail(RESPEC_ERR_INVALID_ARG, "%s: Hq=%d is not a multiple of Hkv=%d", name, p.Hq, p.Hkv);
    if ((dt != RESPEC_F32 && dt != RESPEC_BF16) || (pool_dt != dt && pool_dt != RESPEC_E4M3))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: types %d and %d of the queries and of the pools", name, (int)dt, (int)pool_dt);
    if (pool_dt == RESPEC_E4M3 && dt != RESPEC_BF16) return fail(RESPEC_ERR_UNSUPPORTED, "%s: pools of 8 bits are read by bf16 queries", name);
    if ((pool_dt == RESPEC_E4M3) != (p.k_scale != nullptr) || !p.k_scale != !p.v_scale)
        return fail(RESPEC_ERR_INVALID_ARG, "%s: k_scale and v_scale belong to pools of 8 bits, and only to them", name);
    if (!std::isfinite(sm_scale)) return fail(RESPEC_ERR_INVALID_ARG, "%s: sm_scale must be finite", name);
    if (D != 64 && D != 128) return fail(RESPEC_ERR_UNSUPPORTED, "%s: head size %d is neither 64 nor 128", name, D);
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0)
        return fail(RESPEC_ERR_UNSUPPORTED, "%s: page size %d is not a power of two in [16, 1024]", name, page_size);
    p.max_q = std::min(p.max_q, p.total_q);
    if (!sizes_fit(p.B, p.total_q, p.groups, p.max_q, p.max_kv, p.Hq, p.Hkv, D, dt) || p.B > 65535 || (int64_t)p.Hkv * D * (dt == RESPEC_BF16 ? 2 : 4) > (1 << 24))
        return fail(RESPEC_ERR_UNSUPPORTED, "%s: at most 256 rows and heads to a KV head (G * max_q_per_seq), 65,535 sequences, 2^30 rows and heads", name);
    if (p.tree_mask && p.max_q > 64) return fail(RESPEC_ERR_UNSUPPORTED, "%s: a tree has at most 64 rows", name);
    if (!aligned_to(p.q, 16) || !aligned_to(p.k, 16) || !aligned_to(p.v, 16) || !aligned_to(p.out, 16) || !aligned_to(p.k_scale, 16) || !aligned_to(p.v_scale, 16))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: data pointers and scales must be 16-byte aligned", name);
    const Layout w = layout(p.B, p.total_q, p.groups, p.Hq, D, dt);
    if (!workspace || workspace_bytes < w.bytes || !aligned_to(workspace, 256))
        return fail(RESPEC_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) needed, got %zu", name, w.bytes, workspace ? workspace_bytes : (size_t)0);
    char *const base = static_cast<char *>(workspace);
    p.seq = reinterpret_cast<SeqPlan *>(base + w.seq);
    p.seq_grp = reinterpret_cast<SeqGroup *>(base + w.seq_grp);
    p.grp = reinterpret_cast<GroupPlan *>(base + w.grp);
    p.jobs = reinterpret_cast<Job *>(base + w.jobs);
    p.totals = reinterpret_cast<Totals *>(base + w.totals);
    p.own_o = base + w.own_o;
    p.shared_o = base + w.shared_o;
    p.own_whole_o = base + w.own_whole_o;
    p.shared_whole_o = base + w.shared_whole_o;
    p.own_ml = reinterpret_cast<float *>(base + w.own_ml);
    p.shared_ml = reinterpret_cast<float *>(base + w.shared_ml);
    p.own_whole_ml = reinterpret_cast<float *>(base + w.own_whole_ml);
    p.shared_whole_ml = reinterpret_cast<float *>(base + w.shared_whole_ml);
    p.page_shift = __builtin_ctz((unsigned)page_size);
    p.G = p.Hq / p.Hkv;
    // Columns of a KV head to waves: up to 32 in one, whose neighbours have other heads or keys; more in two (8 bits, as the tiles of two heads fit) or four that
    // share their tiles.
    const int columns = p.G * p.max_q;
    if (pool_dt != RESPEC_E4M3)
        for (p.col_waves = 1; p.col_waves < 4 && p.col_waves * kColumns < columns; p.col_waves *= 2) {}
    else
        p.col_waves = columns <= kColumns ? 1 : columns <= 2 * kColumns && p.Hkv % 2 == 0 ? 2 : 4;
    for (p.heads_wg = 4 / p.col_waves; p.Hkv % p.heads_wg != 0; p.heads_wg /= 2) {}
    p.parts_wg = 4 / (p.col_waves * p.heads_wg);
    p.outer = p.Hkv / p.heads_wg * ((p.G * p.max_q + p.col_waves * kColumns - 1) / (p.col_waves * kColumns));
    for (p.g_shift = 0; (1 << p.g_shift) < p.G; ++p.g_shift) {}
    p.g_mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << p.g_shift) - p.G)) / p.G + 1);
    p.g_shift = std::max(1u, p.g_shift);  // (G = 1 divides nothing)
    const uint32_t sign = dt == RESPEC_BF16 ? 0x80008000u : 0x80000000u;
    p.q_and = sm_scale == 0.f ? 0u : ~0u;
    p.q_xor = sm_scale < 0.f ? sign : 0u;
    p.scale2 = sm_scale == 0.f ? 1.f : (float)(std::fabs((double)sm_scale) * 1.4426950408889634074);
    p.key = 0xcbf29ce484222325u;  // (a plan holds for these sizes only: work-groups that find another's do nothing)
    for (const int64_t x : {(int64_t)p.B, (int64_t)p.groups, (int64_t)p.total_q, (int64_t)p.max_q, (int64_t)p.max_kv, (int64_t)p.num_pages, (int64_t)p.table_len,
                            (int64_t)page_size, (int64_t)p.Hq, (int64_t)p.Hkv, (int64_t)D, (int64_t)dt, (int64_t)pool_dt})
        p.key = (p.key ^ (uint64_t)x) * 0x100000001b3u;
    const Knobs kn = knobs();
    // What a work-group's tile of own keys takes against one of shared keys.  Over bf16 32 groups of 8 sequences at 28/4 heads (two layers) took 178, 163, 162 and
    // 167 us with 130, 165, 220 and 250 hundredths, 64 single tokens 52, 48, 44 and 43; over 8 bits 8 groups of 16 at 40/8 took 165, 157, 166 and 175 us
    // with 130, 160, 200 and 250.
    p.own_cost = (float)std::max(1L, kn.get(&Knobs::shared_cost, pool_dt == RESPEC_E4M3 ? 155 : dt == RESPEC_BF16 ? 220 : 100)) / 100.f;
    // Tiles of own keys that make a range of their own: fp32 takes longer for one than a part more takes to join (8 sequences of up to 40 tokens: 20 us with one,
    // 26 with two), bf16 products do not (8 sequences of 512 to 8,192 tokens at 16/2 heads over 8 bits: 27 us with one, 22 with two, 23 with three).
    p.min_tiles = (int)std::max(1L, kn.get(&Knobs::shared_tiles, dt == RESPEC_F32 ? 1 : 2));
    // What beginning and ending with a sequence's own keys and with a block of columns takes, in tiles.  With none counted the ranges that hold many of them end
    // last: 32 groups of 8 (as above) 177 us, 162 with 1 and 3; 64 single tokens 52 and 44; over 8 bits 8 groups of 16 168 and, with 2 and 3, 157, 256
    // sequences of 512 to 4,096 tokens at 28/4 heads 117 and 109, 96 with trees of seven rows 142 and 130.
    p.own_head = (int)std::max(0L, std::min(kn.get(&Knobs::shared_own_head, pool_dt == RESPEC_BF16 ? 1 : 2), 1000L));
    p.shared_head = (int)std::max(0L, std::min(kn.get(&Knobs::shared_head, 3), 1000L));
    p.max_ranges = (int)std::max(1L, std::min(kn.get(&Knobs::shared_ranges, kJobs), (long)kJobs));
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t err;
    if (pool_dt == RESPEC_E4M3) err = D == 128 ? launch<kE4m3, 128>(p, prepared, stream) : launch<kE4m3, 64>(p, prepared, stream);
    else if (dt == RESPEC_BF16) err = D == 128 ? launch<kBf16, 128>(p, prepared, stream) : launch<kBf16, 64>(p, prepared, stream);
    else err = D == 128 ? launch<kF32, 128>(p, prepared, stream) : launch<kF32, 64>(p, prepared, stream);
    if (err != hipSuccess) return fail(RESPEC_ERR_HIP, "%s: launch failed: %s", name, hipGetErrorString(err));
    clear_error();
    return RESPEC_OK;
}

SharedParams params(const void *q, const void *k_pages, const void *v_pages, const uint8_t *k_scale, const uint8_t *v_scale, const int32_t *q_indptr,
                    const int32_t *page_indptr, const int32_t *page_table, const int32_t *kv_len, const int32_t *group_indptr, const int32_t *shared_len,
                    const uint64_t *tree_mask, void *out, float *lse, int32_t B, int32_t total_q, int32_t num_groups, int32_t num_pages,
                    int32_t page_table_len, int32_t max_q, int32_t max_kv, int32_t Hq, int32_t Hkv) {
    SharedParams p{};
    p.q = static_cast<const char *>(q);
    p.k = static_cast<const char *>(k_pages);
    p.v = static_cast<const char *>(v_pages);
    p.k_scale = k_scale;
    p.v_scale = v_scale;
    p.q_indptr = q_indptr;
    p.page_indptr = page_indptr;
    p.page_table = page_table;
    p.kv_len = kv_len;
    p.group_indptr = group_indptr;
    p.shared_len = shared_len;
    p.tree_mask = tree_mask;
    p.out = static_cast<char *>(out);
    p.lse = lse;
    p.B = B;
    p.groups = num_groups;
    p.total_q = total_q;
    p.max_q = max_q;
    p.max_kv = max_kv;
    p.num_pages = num_pages;
    p.table_len = page_table_len;
    p.Hq = Hq;
    p.Hkv = Hkv;
    return p;
}

}  // namespace
}  // namespace respec

extern "C" {

size_t respec_verify_attention_shared_workspace_bytes(int32_t B, int32_t total_q, int32_t num_groups, int32_t max_q_per_seq, int32_t max_kv_len, int32_t Hq,
                                                      int32_t Hkv, int32_t D, respec_dtype_t dt) {
    using namespace respec;
    if (!sizes_fit(B, total_q, num_groups, std::min(max_q_per_seq, total_q), max_kv_len, Hq, Hkv, D, dt)) return 0;
    return layout(B, total_q, num_groups, Hq, D, dt).bytes;
}

respec_status_t respec_verify_attention_shared(const void *q, const void *k_pages, const void *v_pages, const uint8_t *k_scale, const uint8_t *v_scale,
                                               const int32_t *q_indptr, const int32_t *page_indptr, const int32_t *page_table, const int32_t *kv_len,
                                               const int32_t *group_indptr, const int32_t *shared_len, const uint64_t *tree_mask, void *out, float *lse,
                                               int32_t B, int32_t total_q, int32_t num_groups, int32_t num_pages, int32_t page_table_len,
                                               int32_t page_size, int32_t max_q_per_seq, int32_t max_kv_len, int32_t Hq, int32_t Hkv, int32_t D,
                                               float sm_scale, respec_dtype_t dt, respec_dtype_t pool_dt, void *workspace, size_t workspace_bytes,
                                               void *hip_stream) {
    using namespace respec;
    SharedParams p = params(q, k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table, kv_len, group_indptr, shared_len, tree_mask, out, lse, B,
                            total_q, num_groups, num_pages, page_table_len, max_q_per_seq, max_kv_len, Hq, Hkv);
    return run("verify_attention_shared", p, D, page_size, sm_scale, dt, pool_dt, false, workspace, workspace_bytes, hip_stream);
}

respec_status_t respec_verify_attention_shared_next_layer(const void *q, const void *k_pages, const void *v_pages, const uint8_t *k_scale,
                                                          const uint8_t *v_scale, const int32_t *q_indptr, const int32_t *page_indptr,
                                                          const int32_t *page_table, const int32_t *kv_len, const int32_t *group_indptr,
                                                          const int32_t *shared_len, const uint64_t *tree_mask, void *out, float *lse, int32_t B,
                                                          int32_t total_q, int32_t num_groups, int32_t num_pages, int32_t page_table_len,
                                                          int32_t page_size, int32_t max_q_per_seq, int32_t max_kv_len, int32_t Hq, int32_t Hkv, int32_t D,
                                                          float sm_scale, respec_dtype_t dt, respec_dtype_t pool_dt, void *workspace,
                                                          size_t workspace_bytes, void *hip_stream) {
    using namespace respec;
    SharedParams p = params(q, k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table, kv_len, group_indptr, shared_len, tree_mask, out, lse, B,
                            total_q, num_groups, num_pages, page_table_len, max_q_per_seq, max_kv_len, Hq, Hkv);
    return run("verify_attention_shared_next_layer", p, D, page_size, sm_scale, dt, pool_dt, true, workspace, workspace_bytes, hip_stream);
}

respec_status_t respec_verify_attention_paged_quantised(const void *q, const void *k_pages, const void *v_pages, const uint8_t *k_scale,
                                                        const uint8_t *v_scale, const int32_t *q_indptr, const int32_t *page_indptr,
                                                        const int32_t *page_table, const int32_t *kv_len, const uint64_t *tree_mask, void *out, float *lse,
                                                        int32_t B, int32_t total_q, int32_t num_pages, int32_t page_table_len, int32_t page_size,
                                                        int32_t max_q_per_seq, int32_t max_kv_len, int32_t Hq, int32_t Hkv, int32_t D, float sm_scale,
                                                        respec_dtype_t dt, void *workspace, size_t workspace_bytes, void *hip_stream) {
    using namespace respec;
    SharedParams p = params(q, k_pages, v_pages, k_scale, v_scale, q_indptr, page_indptr, page_table, kv_len, nullptr, nullptr, tree_mask, out, lse, B, total_q, 0,
                            num_pages, page_table_len, max_q_per_seq, max_kv_len, Hq, Hkv);
    return run("verify_attention_paged_quantised", p, D, page_size, sm_scale, dt, RESPEC_E4M3, false, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
