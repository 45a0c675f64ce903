// Verify attention for gfx950 over a paged cache whose sequences share their beginnings, in the cache's type or over a cache of 8 bits.
//
// The responses of a rollout group hold the pages of their prompt together.  The rows of all of them see all the keys that they share, so
// these are a product of many rows (128 to a work-group) with each key and value read once, and only what a sequence holds by itself is read for its own few
// rows.  With (m, l, o) the running maximum, sum and unnormalised output of a part of the keys, the parts are joined by
//     m = max m_i,   l = sum_i l_i 2^(m_i - m),   o = sum_i o_i 2^(m_i - m) / l.
// A work-group does one of the two kinds of work, in one launch: the shared part keeps the matrix cores busy, the other one the memory, and a compute unit
// holds two work-groups.  Both kinds form a flat list of tiles that is cut into even ranges, so every work-group has as much to do whatever the lengths
// are; a range that ends inside a sequence leaves a part, and a second kernel joins the parts in a fixed order.
//
// Products as in the prompt attention: S^T = K Q^T with 32 packed rows (G heads of a KV head to a row) as a wave's columns, the probabilities of a lane's column
// the B operand of O^T = V^T P^T, exponents against a running maximum that moves only where it grows by more than 2^8.
#include "respec_common.hpp"
#include "respec_quantised.hpp"
#include "respec_tiles.hpp"

#include <algorithm>
#include <cmath>

namespace respec {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef s16x4 __attribute__((address_space(3))) *LdsTr;
typedef const __attribute__((address_space(4))) int32_t *ConstInts;  // (read through the scalar cache; nothing writes it meanwhile)

constexpr float kRescaleSlack = 8.f;  // log2 units
constexpr int kWorkGroups = 512;      // two for each compute unit
constexpr int kThreads = 256, kPrepThreads = 1024;
constexpr int kColumns = 32;          // of a wave
constexpr int kBlock = 4 * kColumns;  // columns of a work-group over shared keys
constexpr int kMaxRanges = 4 * kWorkGroups;

struct SeqPlan {
    int64_t base;              // tiles of its own before this sequence's
    int32_t q0, R, L, e0;      // first row, rows, tokens, first entry of page_table
    int32_t shared, group;     // tokens that its group reads for it; -1: none
    int32_t tiles, pad;
};
struct GroupPlan {
    int64_t base;              // tiles of shared keys before this group's
    int32_t q0, rows, shared, e0;
    int32_t key_tiles, blocks; // tiles of keys, blocks of columns
};
struct Start {                 // of a range: its place in the flat list
    int64_t f;
    int32_t outer, item, tile, block;
};
struct Totals {
    int64_t own, shared;       // tiles of an outer step of own work; of a head of shared work
    int32_t shared_wgs, shared_ranges, own_ranges, pad;
    uint64_t key;              // of the sizes that the plan was made for
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
    float shared_cost, own_cost;            // of a work-group's tile, in the same unit
    uint64_t key;
    SeqPlan *seq;
    GroupPlan *grp;
    Start *own_start, *shared_start;
    Totals *totals;
    float *own_o, *own_ml, *shared_o, *shared_ml;                  // parts of ranges' ends
    float *own_whole_o, *own_whole_ml, *shared_whole_o, *shared_whole_ml;  // [total_q * Hq]: parts that are a row's only one of their kind
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
    static constexpr int kOwnKeys = 32, kOwnLoads = kOwnKeys / kLoadKeys, kOwnBytes = 2 * kOwnKeys * kRowBytes;
    static constexpr int kSharedKeys = kHalf ? 64 : 32, kWaveKeys = kSharedKeys / 4;
    static constexpr int kSharedLoads = kWaveKeys / kLoadKeys, kSharedBytes = 2 * kSharedKeys * kRowBytes;
    static constexpr int kLdsBytes = 4 * kOwnBytes > 2 * kSharedBytes ? 4 * kOwnBytes : 2 * kSharedBytes;
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
__device__ inline int64_t block_scan64(int64_t x, int64_t &total, int64_t *lds /* [16] */) {  // exclusive
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t sum = x;
    for (int step = 1; step < 64; step *= 2) {
        const int64_t y = __shfl_up(sum, step);
        if (lane >= step) sum += y;
    }
    if (lane == 63) lds[wave] = sum;
    __syncthreads();
    int64_t before = 0;
    total = 0;
    for (int w = 0; w < kPrepThreads / 64; ++w) {
        before += w < wave ? lds[w] : 0;
        total += lds[w];
    }
    __syncthreads();
    return before + sum - x;
}

// The place of `f` in the flat list: the last item whose base is not past it.
template <typename Item>
__device__ inline int find_item(const Item *items, int n, int64_t f) {
    int at = 0;
    for (int end = n; end - at > 1;) {
        const int mid = (at + end) / 2;
        if (items[mid].base <= f) at = mid;
        else end = mid;
    }
    return at;
}

// One work-group reads the index arrays and writes what every other one needs: what each sequence and group has to do, and where the ranges begin.
template <int SHARED_KEYS>
__global__ __launch_bounds__(kPrepThreads) void shared_prep_kernel(SharedParams p) {
    __shared__ int64_t lds[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = threadIdx.x; b < p.B; b += kPrepThreads) {
        SeqPlan s{};
        s.q0 = max(0, min(p.q_indptr[b], p.total_q));
        s.R = max(0, min(min(p.q_indptr[b + 1], p.total_q) - s.q0, p.max_q));
        s.e0 = max(0, min(p.page_indptr[b], p.table_len));
        const int64_t held = max(0, min(p.page_indptr[b + 1], p.table_len) - s.e0);
        s.L = (int)max((int64_t)0, min(min((int64_t)p.kv_len[b], held << p.page_shift), (int64_t)p.max_kv));
        s.group = -1;
        p.seq[b] = s;
    }
    __syncthreads();
    for (int g = wave; g < p.groups; g += kPrepThreads / 64) {  // a wave per group: what all its members hold before their new tokens
        const int first = max(0, min(p.group_indptr[g], p.B)), end = max(first, min(p.group_indptr[g + 1], p.B));
        int shared = end - first < 2 ? 0 : p.shared_len[g];
        for (int b = first + lane; b < end; b += 64) shared = min(shared, p.seq[b].L - p.seq[b].R);
        for (int step = 1; step < 64; step *= 2) shared = min(shared, __shfl_xor(shared, step));
        shared = max(0, shared);
        GroupPlan t{};
        if (shared > 0) {
            t.q0 = p.seq[first].q0;
            t.rows = max(0, p.seq[end - 1].q0 + p.seq[end - 1].R - t.q0);
            t.e0 = p.seq[first].e0;
            t.shared = t.rows > 0 ? shared : 0;
            t.key_tiles = (t.shared + SHARED_KEYS - 1) / SHARED_KEYS;
            t.blocks = (int)(((int64_t)t.rows * p.G + kBlock - 1) / kBlock);
        }
        if (lane == 0) p.grp[g] = t;
        if (t.shared > 0)
            for (int b = first + lane; b < end; b += 64) {
                p.seq[b].shared = t.shared;
                p.seq[b].group = g;
            }
    }
    __syncthreads();
    int64_t own = 0, shared = 0, total;
    for (int b0 = 0; b0 < p.B; b0 += kPrepThreads) {
        const int b = b0 + threadIdx.x;
        int tiles = 0;
        if (b < p.B) {
            const SeqPlan s = p.seq[b];
            if (s.R > 0 && s.L > s.shared) tiles = (int)(((int64_t)s.L + 31) / 32) - s.shared / 32;
        }
        const int64_t base = own + block_scan64(tiles, total, lds);
        if (b < p.B) {
            p.seq[b].base = base;
            p.seq[b].tiles = tiles;
        }
        own += total;
    }
    for (int g0 = 0; g0 < p.groups; g0 += kPrepThreads) {
        const int g = g0 + threadIdx.x;
        const int64_t n = g < p.groups ? (int64_t)p.grp[g].key_tiles * p.grp[g].blocks : 0;
        const int64_t base = shared + block_scan64(n, total, lds);
        if (g < p.groups) p.grp[g].base = base;
        shared += total;
    }
    // Work-groups for each kind by what its tiles cost, whole eights of them (the XCDs take turns), at least a few tiles to a range.
    const int64_t all_own = own * p.outer, all_shared = shared * p.Hkv;
    const float cost_s = (float)all_shared * p.shared_cost, cost_o = (float)all_own / p.parts_wg * p.own_cost;
    Totals t{};
    t.own = own;
    t.shared = shared;
    if (all_shared > 0) {
        const int even = (int)(kWorkGroups / 8 * (cost_s / (cost_s + cost_o)) + 0.5f) * 8;
        t.shared_wgs = all_own > 0 ? max(8, min(even, kWorkGroups - 8)) : kWorkGroups;
        t.shared_ranges = (int)min((int64_t)t.shared_wgs, (all_shared + 1) / 2);
    }
    t.own_ranges = (int)min((int64_t)(kWorkGroups - t.shared_wgs) * p.parts_wg, (all_own + 3) / 4);
    t.key = p.key;
    if (threadIdx.x == 0) *p.totals = t;
    __syncthreads();
    for (int r = threadIdx.x; r <= t.own_ranges; r += kPrepThreads) {
        Start s{};
        s.f = t.own_ranges == 0 ? 0 : (int64_t)(((__int128)all_own * r) / t.own_ranges);
        if (r < t.own_ranges) {
            s.outer = (int)(s.f / own);
            const int64_t rest = s.f - s.outer * own;
            s.item = find_item(p.seq, p.B, rest);
            s.tile = (int)(rest - p.seq[s.item].base);
        }
        p.own_start[r] = s;
    }
    for (int r = threadIdx.x; r <= t.shared_ranges; r += kPrepThreads) {
        Start s{};
        s.f = t.shared_ranges == 0 ? 0 : (int64_t)(((__int128)all_shared * r) / t.shared_ranges);
        if (r < t.shared_ranges) {
            s.outer = (int)(s.f / shared);
            const int64_t rest = s.f - s.outer * shared;
            s.item = find_item(p.grp, p.groups, rest);
            const GroupPlan g = p.grp[s.item];
            const int64_t in = rest - g.base;
            s.block = (int)(in / g.key_tiles);
            s.tile = (int)(in - (int64_t)s.block * g.key_tiles);
        }
        p.shared_start[r] = s;
    }
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
    // Q^T as the B operand: a lane's column is its row, its contraction slots the pieces 2x + half of the row.
    __device__ void load_q(const SharedParams &p, int64_t row, int head, int half) {
        const char *from = p.q + (row * p.Hq + head) * (int64_t)S::kRowBytes + half * 16;
#pragma unroll
        for (int x = 0; x < S::kPieces / 2; ++x) {
            qf[x] = *reinterpret_cast<const u32x4 *>(from + x * 32);
            for (int w = 0; w < 4; ++w) qf[x][w] = (qf[x][w] & p.q_and) ^ p.q_xor;
        }
    }
};

// A tile of NB blocks of 32 keys in LDS (K at `k`, V at `v`): the scores, masked by `mask` (scores of a block, its number), into the state.
template <Pool POOL, int D, int NB, typename Mask>
__device__ __attribute__((always_inline)) inline void attend(const SharedParams &p, State<POOL, D> &st, const char *lds, int k, int v, int half, int col, Mask &&mask) {
    using S = Shape<POOL, D>;
    floatx16 s[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        for (int x = 0; x < 16; ++x) s[b][x] = 0.f;
#pragma unroll
        for (int x = 0; x < S::kPieces / 2; ++x) {
            const u32x4 a = *reinterpret_cast<const u32x4 *>(lds + k + (b * 32 + col) * S::kRowBytes + k_piece<S::kHalf, D>(col, 2 * x + half) * 16);
            if constexpr (S::kHalf) {
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, st.qf[x]), s[b], 0, 0, 0);
            } else {
#pragma unroll
                for (int y = 0; y < 4; ++y) s[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[y]), __uint_as_float(st.qf[x][y]), s[b], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) mask(s[b], b);
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int x = 0; x < 16; ++x) top = fmaxf(top, s[b][x]);
    top = max_of_halves(top) * p.scale2;
    if (__ballot(top > st.m + kRescaleSlack) != 0) {  // (m = -inf: any finite score)
        const float m_new = top > st.m + kRescaleSlack ? top : st.m;
        const float f = st.m == m_new ? 1.f : __builtin_amdgcn_exp2f(st.m - m_new);
        st.m = m_new;
        st.ref = m_new == -INFINITY ? 0.f : m_new;
        st.l *= f;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
            for (int x = 0; x < 16; ++x) st.o[d][x] *= f;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            s[b][x] = __builtin_amdgcn_exp2f(fmaf(s[b][x], p.scale2, -st.ref));
            st.l += s[b][x];
        }
    if constexpr (S::kHalf) {
        // V by transposing reads: sixteen lanes address four keys by sixteen d and receive one d of the four keys each.
        const int lane = half * 32 + col, i16 = lane & 15, v_key = half * 4 + (i16 >> 2), d0 = ((lane & 16) + 4 * (i16 & 3)) * 2;
        const int v_at = v + v_key * S::kRowBytes + v_piece<true, D>(v_key, d0 >> 4) * 16 + (d0 & 15);
#pragma unroll
        for (int g = 0; g < 2 * NB; ++g) {  // sixteen keys at a time: slot j is key 8 (j / 4) + 4 half + j % 4 of them; their probabilities rounded to bf16
            u32x4 pf;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                pf[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{s[g / 2][g % 2 * 8 + 2 * j], s[g / 2][g % 2 * 8 + 2 * j + 1]}, bf16x2));
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
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const int key = b * 32 + 8 * (x / 4) + 4 * half + x % 4;
#pragma unroll
                for (int d = 0; d < S::kDTiles; ++d)
                    st.o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float *>(lds + v + key * S::kRowBytes + (d * 32 + col) * 4), s[b][x], st.o[d], 0, 0, 0);
            }
    }
}

// A wave's keys on their way from the pools through registers into LDS.  Its loads cover aligned runs of sixteen keys, each within a page; what
// differs between lanes is a 32-bit offset.  Keys past the last one (`left` behind a run's first) are the last one's: they are never seen.
enum Put { kAll = 0, kCut = 1, kSift = 2 };
template <Pool POOL, int D, int LOADS>
struct Mover {
    using S = Shape<POOL, D>;
    u32x4 k[LOADS], v[LOADS];
    uint32_t ks[POOL == kE4m3 ? LOADS : 1], vs[POOL == kE4m3 ? LOADS : 1];
    // Runs of `per_run` loads from key n0 on (a multiple of sixteen, or eight behind one), head h; the sequence's entries begin at e0, its last key is `last`.
    template <bool NT>
    __device__ __attribute__((always_inline)) inline void load(const SharedParams &p, int e0, int h, int n0, int last, int lane) {
        constexpr int kRun = (16 / S::kLoadKeys) < LOADS ? 16 / S::kLoadKeys : LOADS;
        const ConstInts table = (ConstInts)p.page_table;
        const int my_key = lane / S::kPoolPieces;
        const uint32_t piece = (uint32_t)(lane % S::kPoolPieces) * 16, token = (uint32_t)p.Hkv * D * S::kPoolSize;
#pragma unroll
        for (int run = 0; run < LOADS / kRun; ++run) {
            const int n = min(n0 + run * 16, last);
            const int64_t page = max(0, min(table[e0 + (n >> p.page_shift)], p.num_pages - 1));
            const int slot = n & ((1 << p.page_shift) - 1), left = last - n;
            const int64_t row = ((page << p.page_shift) + slot) * p.Hkv + h;
            const char *kp = p.k + row * (D * S::kPoolSize), *vp = p.v + row * (D * S::kPoolSize);
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                const int i = run * kRun + j, key = min(j * S::kLoadKeys + my_key, left);
                const uint32_t off = (uint32_t)key * token + piece;
                const u32x4 *a = reinterpret_cast<const u32x4 *>(kp + off), *b = reinterpret_cast<const u32x4 *>(vp + off);
                k[i] = NT ? __builtin_nontemporal_load(a) : *a;
                v[i] = NT ? __builtin_nontemporal_load(b) : *b;
                if constexpr (POOL == kE4m3) {
                    const int64_t at = ((page * p.Hkv + h) << p.page_shift) + slot + key;
                    ks[i] = p.k_scale[at];
                    vs[i] = p.v_scale[at];
                }
            }
        }
    }
    // Into the rows `key0` on of a tile.  kCut: V of keys outside [begin, end) is zero.  kSift: also, some row does not see all of these keys.  A product would
    // carry a value of V that is not finite to it all the same, so such values count as zero here; they are added at the end to the rows that see them.
    template <Put SIFT>
    __device__ __attribute__((always_inline)) inline bool put(char *kt, char *vt, int key0, int lane, int n0, int begin, int end) {
        const int my_key = lane / S::kPoolPieces, piece = lane % S::kPoolPieces;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int key = key0 + i * S::kLoadKeys + my_key;
            constexpr int kOut = POOL == kE4m3 ? 2 : 1;
            u32x4 a[kOut], b[kOut];
            if constexpr (POOL == kE4m3) {
                const float sk = scale_of((int)ks[i]), sv = scale_of((int)vs[i]);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t lo, hi;
                    values_of(k[i][w], sk, lo, hi);
                    a[w / 2][w % 2 * 2] = lo;
                    a[w / 2][w % 2 * 2 + 1] = hi;
                    values_of(v[i][w], sv, lo, hi);
                    b[w / 2][w % 2 * 2] = lo;
                    b[w / 2][w % 2 * 2 + 1] = hi;
                }
            } else {
                a[0] = k[i];
                b[0] = v[i];
            }
            if constexpr (SIFT != kAll) {
                const int n = n0 + i * S::kLoadKeys + my_key;
                const bool none = n < begin || n >= end;
#pragma unroll
                for (int y = 0; y < kOut; ++y)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const bool hi = SIFT == kSift && (b[y][w] & 0x7f800000u) == 0x7f800000u, lo = SIFT == kSift && S::kHalf && (b[y][w] & 0x7f80u) == 0x7f80u;
                        bad |= (hi || lo) && !none;
                        b[y][w] &= none ? 0u : (hi ? (S::kHalf ? 0xffffu : 0u) : ~0u) & (lo ? 0xffff0000u : ~0u);
                    }
            }
#pragma unroll
            for (int y = 0; y < kOut; ++y) {
                *reinterpret_cast<u32x4 *>(kt + key * S::kRowBytes + k_piece<S::kHalf, D>(key, piece * kOut + y) * 16) = a[y];
                *reinterpret_cast<u32x4 *>(vt + key * S::kRowBytes + v_piece<S::kHalf, D>(key, piece * kOut + y) * 16) = b[y];
            }
        }
        return bad;
    }
};

// A wave's columns as a part: unnormalised output, maximum and sum.  `o`, `ml`: of the lane's column.
template <Pool POOL, int D>
__device__ inline void write_part(const State<POOL, D> &st, float l, float *o, float *ml, bool exists, int half) {
    if (!exists) return;
    if (half == 0) *reinterpret_cast<floatx2 *>(ml) = floatx2{st.m, l};
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int x = 0; x < 16; x += 4)
            *reinterpret_cast<floatx4 *>(o + d * 32 + 2 * x + 4 * half) = floatx4{st.o[d][x], st.o[d][x + 1], st.o[d][x + 2], st.o[d][x + 3]};
}

// ------------------------------------------------------------------------------------------ keys that a group shares
// Every wave has 32 of the work-group's 128 columns; the four stage a tile of keys together, into one of two places in LDS while the other is read.
template <Pool POOL, int D>
__device__ __attribute__((always_inline)) inline void shared_work(const SharedParams &p, char *lds, int r) {
    using S = Shape<POOL, D>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    Start at = p.shared_start[r];
    const int64_t f0 = at.f, f1 = p.shared_start[r + 1].f;
    if (f0 >= f1) return;
    GroupPlan g = p.grp[at.item];
    State<POOL, D> st;
    Mover<POOL, D, S::kSharedLoads> mover;
    auto fetch = [&]() __attribute__((always_inline)) {
        mover.template load<false>(p, g.e0, at.outer, at.tile * S::kSharedKeys + wave * S::kWaveKeys, g.shared - 1, lane);
    };
    auto put = [&](int place) __attribute__((always_inline)) {
        const int n0 = at.tile * S::kSharedKeys;
        char *const kt = lds + place * S::kSharedBytes, *const vt = kt + S::kSharedBytes / 2;
        // (all rows see all keys: what is not finite goes where it belongs, only what lies past the keys is left out)
        if (n0 + S::kSharedKeys <= g.shared) mover.template put<kAll>(kt, vt, wave * S::kWaveKeys, lane, 0, 0, 0);
        else mover.template put<kCut>(kt, vt, wave * S::kWaveKeys, lane, n0 + wave * S::kWaveKeys, 0, g.shared);
    };
    fetch();
    put(0);
    int place = 0;
    bool fresh = true, first = true;
    int64_t row = 0;
    int head = 0, column = 0;
    bool exists = false;
    for (int64_t f = f0; f < f1; ++f) {
        const Start now = at;
        const GroupPlan gn = g;
        if (fresh) {
            column = now.block * kBlock + wave * kColumns + col;
            exists = column < gn.rows * p.G;
            const int c = min(column, gn.rows * p.G - 1), i = by_g(p, c);
            row = gn.q0 + i;
            head = now.outer * p.G + c - i * p.G;
            st.clear();
            st.load_q(p, row, head, half);
            fresh = false;
        }
        if (++at.tile == g.key_tiles) {  // the next tile's place
            at.tile = 0;
            if (++at.block == g.blocks) {
                at.block = 0;
                if (f + 1 < f1) {
                    do {
                        if (++at.item == p.groups) {
                            at.item = 0;
                            ++at.outer;
                        }
                    } while (p.grp[at.item].key_tiles == 0);
                    g = p.grp[at.item];
                }
            }
            fresh = true;
        }
        if (f + 1 < f1) fetch();
        __syncthreads();  // (this tile is there, and the other place has been read)
        if (now.block * kBlock + wave * kColumns < gn.rows * p.G) {
            const int n0 = now.tile * S::kSharedKeys;
            const bool cut = n0 + S::kSharedKeys > gn.shared;
            attend<POOL, D, S::kSharedKeys / 32>(p, st, lds, place * S::kSharedBytes, place * S::kSharedBytes + S::kSharedBytes / 2, half, col,
                                                 [&](floatx16 &s, int b) __attribute__((always_inline)) {
                                                     if (!cut) return;
#pragma unroll
                                                     for (int x = 0; x < 16; ++x)
                                                         if (n0 + b * 32 + 8 * (x / 4) + 4 * half + x % 4 >= gn.shared) s[x] = -INFINITY;
                                                 });
        }
        place ^= 1;
        if (f + 1 < f1) put(place);
        if (fresh || f + 1 == f1) {
            const bool whole = now.tile + 1 == gn.key_tiles && f - now.tile >= f0;
            const float l = sum_of_halves(st.l);
            const int64_t index = whole ? row * p.Hq + head : ((int64_t)2 * r + !first) * kBlock + wave * kColumns + col;
            write_part<POOL, D>(st, l, (whole ? p.shared_whole_o : p.shared_o) + index * D, (whole ? p.shared_whole_ml : p.shared_ml) + index * 2, exists, half);
            first = false;
        }
    }
}

// ------------------------------------------------------------------------------------------ keys of a sequence by itself
// Every wave walks a range of its own, without barriers: tiles of 32 keys, the next one on its way into registers while this one is read from the
// wave's part of LDS.  Neighbouring waves have neighbouring KV heads of the same keys.
template <Pool POOL, int D>
__device__ __attribute__((always_inline)) inline void own_work(const SharedParams &p, char *lds, int wg) {
    using S = Shape<POOL, D>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    const int cw = wave % p.col_waves, hi = wave / p.col_waves % p.heads_wg, part = wave / (p.col_waves * p.heads_wg);
    const int r = wg * p.parts_wg + part;
    if (r >= p.totals->own_ranges) return;
    Start at = p.own_start[r];
    const int64_t f0 = at.f, f1 = p.own_start[r + 1].f;
    if (f0 >= f1) return;
    const int head_groups = p.Hkv / p.heads_wg;
    char *const kt = lds + wave * S::kOwnBytes, *const vt = kt + S::kOwnBytes / 2;
    SeqPlan s = p.seq[at.item];
    State<POOL, D> st;
    Mover<POOL, D, S::kOwnLoads> mover;
    auto fetch = [&]() __attribute__((always_inline)) {
        mover.template load<true>(p, s.e0, at.outer % head_groups * p.heads_wg + hi, (s.shared / 32 + at.tile) * 32, s.L - 1, lane);
    };
    fetch();
    bool fresh = true, first = true, bad = false, exists = false;
    int64_t row = 0;
    int head = 0, lim = 0, packed0 = 0, begin_tile = 0;
    uint64_t bits = 0;
    for (int64_t f = f0; f < f1; ++f) {
        const Start now = at;
        const SeqPlan sn = s;
        const int kv_head = now.outer % head_groups * p.heads_wg + hi;
        const int n0 = (sn.shared / 32 + now.tile) * 32, before = sn.L - sn.R;  // keys before the new tokens (negative: the first rows see none)
        const bool special = n0 < sn.shared || n0 + 32 > before + (p.tree_mask ? 0 : 1);
        if (special) bad |= mover.template put<kSift>(kt, vt, 0, lane, n0, sn.shared, sn.L);
        else mover.template put<kAll>(kt, vt, 0, lane, 0, 0, 0);
        if (fresh) {
            packed0 = (now.outer / head_groups * p.col_waves + cw) * kColumns;
            begin_tile = now.tile;
            const int last = sn.R * p.G - 1, c = min(packed0 + col, last), i = by_g(p, c);
            exists = packed0 + col <= last;
            row = sn.q0 + i;
            head = kv_head * p.G + c - i * p.G;
            lim = before + i + 1;
            if (p.tree_mask) bits = p.tree_mask[row];
            st.clear();
            st.load_q(p, row, head, half);
            fresh = false;
        }
        if (++at.tile == s.tiles) {
            at.tile = 0;
            if (f + 1 < f1) {
                do {
                    if (++at.item == p.B) {
                        at.item = 0;
                        ++at.outer;
                    }
                } while (p.seq[at.item].tiles == 0);
                s = p.seq[at.item];
            }
            fresh = true;
        }
        if (f + 1 < f1) fetch();
        wave_sync();
        if (packed0 < sn.R * p.G)  // (uniform)
            attend<POOL, D, 1>(p, st, lds, wave * S::kOwnBytes, wave * S::kOwnBytes + S::kOwnBytes / 2, half, col, [&](floatx16 &sc, int) __attribute__((always_inline)) {
                if (!special) return;
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    const int n = n0 + 8 * (x / 4) + 4 * half + x % 4;
                    const bool sees = p.tree_mask ? n < before || (n < sn.L && n - before < 64 && (bits >> (n - before) & 1)) : n < lim;
                    if (n < sn.shared || !sees) sc[x] = -INFINITY;
                }
            });
        wave_sync();
        if (!fresh && f + 1 < f1) continue;
        const bool whole = begin_tile == 0 && now.tile + 1 == sn.tiles, final = whole && sn.shared == 0;
        const float l = sum_of_halves(st.l);
        const int64_t index = whole ? row * p.Hq + head : (((int64_t)2 * r + !first) * (4 / p.parts_wg) + hi * p.col_waves + cw) * kColumns + col;
        float *const part_o = (whole ? p.own_whole_o : p.own_o) + index * D, *const part_ml = (whole ? p.own_whole_ml : p.own_ml) + index * 2;
        if (final) {  // all that the row sees
            const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;  // (no visible key: zero; NaN stays)
            char *const to = p.out + (row * p.Hq + head) * (int64_t)S::kRowBytes;
            if (exists) {
                if (p.lse && half == 0) p.lse[row * p.Hq + head] = l == 0.f ? -INFINITY : st.m * 0.693147180559945309f + logf(l);
#pragma unroll
                for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
                    for (int x = 0; x < 16; x += 4) {
                        const floatx4 y = {st.o[d][x] * inv, st.o[d][x + 1] * inv, st.o[d][x + 2] * inv, st.o[d][x + 3] * inv};
                        if constexpr (S::kHalf) {
                            const bf16x2 a = __builtin_convertvector(floatx2{y[0], y[1]}, bf16x2), b = __builtin_convertvector(floatx2{y[2], y[3]}, bf16x2);
                            *reinterpret_cast<u32x2 *>(to + (d * 32 + 2 * x + 4 * half) * 2) = u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
                        } else {
                            *reinterpret_cast<floatx4 *>(to + (d * 32 + 2 * x + 4 * half) * 4) = y;
                        }
                    }
            }
        } else {
            write_part<POOL, D>(st, l, part_o, part_ml, exists, half);
        }
        first = false;
        if (__ballot(bad) != 0) {
            // The values that put() left out, added to what this wave has written: a column and a d of it per lane.
            bad = false;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
            __builtin_amdgcn_wave_barrier();
            // (in the tile that the shared keys end in, and from the first one on that some row does not see all of)
            const int first_key = (sn.shared / 32 + begin_tile) * 32, end_key = min(n0 + 32, sn.L);
            const int next = first_key < sn.shared ? first_key + 32 : first_key, masked = max(next, max(before, 0) / 32 * 32);
            for (int e = lane; e < kColumns * D; e += 64) {
                const int c = packed0 + e / D, d = e % D;
                if (c >= sn.R * p.G) break;
                const int i = by_g(p, c);
                const uint64_t own_bits = p.tree_mask ? p.tree_mask[sn.q0 + i] : 0;
                float sum = 0.f;
                for (int n = first_key < sn.shared ? sn.shared : masked; n < end_key; n = n + 1 == next ? masked : n + 1) {
                    const bool sees = p.tree_mask ? n < before || (n - before < 64 && (own_bits >> (n - before) & 1)) : n <= before + i;
                    if (!sees) continue;
                    const int64_t page = max(0, min(p.page_table[sn.e0 + (n >> p.page_shift)], p.num_pages - 1));
                    const int slot = n & ((1 << p.page_shift) - 1);
                    const int64_t el = (((page << p.page_shift) + slot) * p.Hkv + kv_head) * D + d;
                    float x;
                    if constexpr (POOL == kF32) x = reinterpret_cast<const float *>(p.v)[el];
                    else if constexpr (POOL == kBf16) x = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(p.v)[el] << 16);
                    else {
                        uint32_t lo, hi;
                        values_of(reinterpret_cast<const uint8_t *>(p.v)[el], scale_of(p.v_scale[((page * p.Hkv + kv_head) << p.page_shift) + slot]), lo, hi);
                        x = __uint_as_float(lo << 16);
                    }
                    if (!(fabsf(x) < INFINITY)) sum += x;
                }
                if (sum == 0.f) continue;
                const int64_t q_row = sn.q0 + i, q_head = kv_head * p.G + c - i * p.G;
                if (final) {
                    char *const to = p.out + ((q_row * p.Hq + q_head) * D + d) * S::kSize;
                    if constexpr (S::kHalf) *reinterpret_cast<uint16_t *>(to) = __builtin_bit_cast(uint16_t, (__bf16)(__uint_as_float((uint32_t)*reinterpret_cast<uint16_t *>(to) << 16) + sum));
                    else *reinterpret_cast<float *>(to) += sum;
                } else {
                    const int64_t at_col = whole ? q_row * p.Hq + q_head : index - col + e / D;
                    (whole ? p.own_whole_o : p.own_o)[at_col * D + d] += sum;
                }
            }
        }
    }
}

template <Pool POOL, int D>
__global__ __launch_bounds__(kThreads, POOL == kF32 ? 1 : 2) void shared_attention_kernel(SharedParams p) {
    extern __shared__ __align__(16) char lds[];
    if (p.totals->key != p.key) return;  // (no plan of these sizes)
    const int wgs = __builtin_amdgcn_readfirstlane(p.totals->shared_wgs), wg = blockIdx.x;
    if (wg < wgs) {
        // consecutive ranges, which read the same keys for other columns, on one XCD (work-groups go to the XCDs in turn)
        const int r = wg % 8 * (wgs / 8) + wg / 8;
        if (r < p.totals->shared_ranges) shared_work<POOL, D>(p, lds, r);
    } else {
        own_work<POOL, D>(p, lds, wg - wgs);
    }
}

// ------------------------------------------------------------------------------------------ joining the parts
// The range whose tiles include f.
__device__ inline int range_of(const Start *start, int n, int64_t total, int64_t f) {
    int r = max(0, min(n - 1, (int)((double)f * n / (double)total)));
    while (r > 0 && start[r].f > f) --r;
    while (r + 1 < n && start[r + 1].f <= f) ++r;
    return r;
}

// D / 4 lanes for each row and head of a sequence.
template <bool HALF, int D>
__global__ __launch_bounds__(kThreads) void shared_join_kernel(SharedParams p) {
    constexpr int kQuads = D / 4, kPer = kThreads / kQuads;
    const Totals t = *p.totals;
    if (t.key != p.key) return;
    const SeqPlan s = p.seq[blockIdx.y];
    const int item = blockIdx.x * kPer + threadIdx.x / kQuads, quad = threadIdx.x % kQuads;
    if (item >= s.R * p.Hq) return;
    const int i = item / p.Hq, head = item % p.Hq, kv_head = head / p.G, c = i * p.G + head % p.G;
    const int64_t row = s.q0 + i, at = row * p.Hq + head;
    float m = -INFINITY, l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](const float *part_o, const float *part_ml, int64_t index) __attribute__((always_inline)) {
        const floatx2 ml = *reinterpret_cast<const floatx2 *>(part_ml + index * 2);
        const floatx4 x = *reinterpret_cast<const floatx4 *>(part_o + index * D + quad * 4);
        if (ml[1] == 0.f) return;  // (no key of this part is seen)
        const float m_new = fmaxf(m, ml[0]);
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new), e = __builtin_amdgcn_exp2f(ml[0] - m_new);
        l = l * f + ml[1] * e;
        for (int j = 0; j < 4; ++j) o[j] = o[j] * f + x[j] * e;
        m = m_new;
    };
    if (s.shared > 0) {
        const GroupPlan g = p.grp[s.group];
        const int packed = max(0, min((int)(row - g.q0) * p.G + head % p.G, g.rows * p.G - 1)), block = packed / kBlock;
        const int64_t all = t.shared * p.Hkv, b = t.shared * kv_head + g.base + (int64_t)block * g.key_tiles, e = b + g.key_tiles - 1;
        const int r0 = range_of(p.shared_start, t.shared_ranges, all, b), r1 = range_of(p.shared_start, t.shared_ranges, all, e);
        if (r0 == r1) add(p.shared_whole_o, p.shared_whole_ml, at);
        else
            for (int r = r0; r <= r1; ++r) add(p.shared_o, p.shared_ml, ((int64_t)2 * r + (r == r0 && p.shared_start[r].f < b)) * kBlock + packed % kBlock);
    }
    if (s.tiles > 0) {
        const int cols = p.col_waves * kColumns, hi = kv_head % p.heads_wg, outer = c / cols * (p.Hkv / p.heads_wg) + kv_head / p.heads_wg;
        const int64_t all = t.own * p.outer, b = t.own * outer + s.base, e = b + s.tiles - 1;
        const int r0 = range_of(p.own_start, t.own_ranges, all, b), r1 = range_of(p.own_start, t.own_ranges, all, e);
        if (r0 == r1) {
            if (s.shared == 0) return;  // (written already)
            add(p.own_whole_o, p.own_whole_ml, at);
        } else {
            for (int r = r0; r <= r1; ++r)
                add(p.own_o, p.own_ml, (((int64_t)2 * r + (r == r0 && p.own_start[r].f < b)) * (4 / p.parts_wg) + hi * p.col_waves + c % cols / kColumns) * kColumns + c % kColumns);
        }
    }
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    for (int j = 0; j < 4; ++j) o[j] *= inv;
    if constexpr (HALF) {
        const bf16x2 a = __builtin_convertvector(floatx2{o[0], o[1]}, bf16x2), b = __builtin_convertvector(floatx2{o[2], o[3]}, bf16x2);
        *reinterpret_cast<u32x2 *>(p.out + (at * D + quad * 4) * 2) = u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    } else {
        *reinterpret_cast<floatx4 *>(p.out + (at * D + quad * 4) * 4) = o;
    }
    if (p.lse && quad == 0) p.lse[at] = l == 0.f ? -INFINITY : m * 0.693147180559945309f + logf(l);
}

// ------------------------------------------------------------------------------------------ host side
// The workspace, piece by piece, each at a multiple of 256 bytes.
struct Layout {
    size_t seq, grp, own_start, shared_start, totals, own_o, own_ml, shared_o, shared_ml, own_whole_o, own_whole_ml, shared_whole_o, shared_whole_ml, bytes;
};
Layout layout(int32_t B, int32_t total_q, int32_t groups, int32_t Hq, int32_t D) {
    Layout w{};
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t here = at;
        at += round_up(n, 256);
        return here;
    };
    const size_t f = sizeof(float), rows = (size_t)total_q * Hq, own = (size_t)kWorkGroups * 8 * kColumns, shared = groups > 0 ? (size_t)kWorkGroups * 2 * kBlock : 0;
    w.seq = take((size_t)B * sizeof(SeqPlan));
    w.grp = take((size_t)groups * sizeof(GroupPlan));
    w.own_start = take((kMaxRanges + 1) * sizeof(Start));
    w.shared_start = take((kWorkGroups + 1) * sizeof(Start));
    w.totals = take(sizeof(Totals));
    w.own_ml = take(own * 2 * f);
    w.own_o = take(own * D * f);
    w.shared_ml = take(shared * 2 * f);
    w.shared_o = take(shared * D * f);
    if (groups > 0) {
        w.own_whole_ml = take(rows * 2 * f);
        w.own_whole_o = take(rows * D * f);
        w.shared_whole_ml = take(rows * 2 * f);
        w.shared_whole_o = take(rows * D * f);
    }
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
    if (!prepared) hipLaunchKernelGGL(shared_prep_kernel<S::kSharedKeys>, dim3(1), dim3(kPrepThreads), 0, stream, p);
    auto *kernel = &shared_attention_kernel<POOL, D>;
    if (S::kLdsBytes > 65536) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::kLdsBytes);
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL(kernel, dim3(kWorkGroups), dim3(kThreads), S::kLdsBytes, stream, p);
    constexpr int kPer = kThreads / (D / 4);
    hipLaunchKernelGGL((shared_join_kernel<S::kHalf, D>), dim3((unsigned)((p.max_q * p.Hq + kPer - 1) / kPer), (unsigned)p.B), dim3(kThreads), 0, stream, p);
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
    if (!aligned_to(p.q, 16) || !aligned_to(p.k, 16) || !aligned_to(p.v, 16) || !aligned_to(p.out, 16))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: data pointers must be 16-byte aligned", name);
    const Layout w = layout(p.B, p.total_q, p.groups, p.Hq, D);
    if (!workspace || workspace_bytes < w.bytes || !aligned_to(workspace, 256))
        return fail(RESPEC_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) needed, got %zu", name, w.bytes, workspace ? workspace_bytes : (size_t)0);
    char *const base = static_cast<char *>(workspace);
    p.seq = reinterpret_cast<SeqPlan *>(base + w.seq);
    p.grp = reinterpret_cast<GroupPlan *>(base + w.grp);
    p.own_start = reinterpret_cast<Start *>(base + w.own_start);
    p.shared_start = reinterpret_cast<Start *>(base + w.shared_start);
    p.totals = reinterpret_cast<Totals *>(base + w.totals);
    for (const auto &[to, at] : {std::pair<float **, size_t>{&p.own_o, w.own_o}, {&p.own_ml, w.own_ml}, {&p.shared_o, w.shared_o}, {&p.shared_ml, w.shared_ml},
                                 {&p.own_whole_o, w.own_whole_o}, {&p.own_whole_ml, w.own_whole_ml}, {&p.shared_whole_o, w.shared_whole_o}, {&p.shared_whole_ml, w.shared_whole_ml}})
        *to = reinterpret_cast<float *>(base + at);
    p.page_shift = __builtin_ctz((unsigned)page_size);
    p.G = p.Hq / p.Hkv;
    for (p.col_waves = 1; p.col_waves < 4 && p.col_waves * kColumns < p.G * p.max_q; p.col_waves *= 2) {}
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
    p.shared_cost = 1.f;
    p.own_cost = pool_dt == RESPEC_E4M3 ? 0.7f : 1.f;
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
    return layout(B, total_q, num_groups, Hq, D).bytes;
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
