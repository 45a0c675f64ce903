// Attention over whole prompts for gfx950: causal, grouped-query heads, packed sequences of different lengths, keys and values in one
// piece or in pages.  This is the forward that fills a cache before the drafts begin and rebuilds it when a sequence moves between
// speculative and plain decoding (Section 5.2); a prompt may come in chunks, its earlier tokens being in the cache already.
//
// The G query heads of a KV head are packed into the rows: packed row r is row r / G, head r % G, so a tile of 128 or 256
// rows spans that many over G positions, reads K and V once for all its heads and wastes little on the diagonal or on a short prompt.  A wave holds 32
// packed rows as the columns of 32x32 MFMA tiles (v_mfma_f32_32x32x16_bf16, v_mfma_f32_32x32x2_f32): S^T = K Q^T leaves a
// lane's scores in one column, so the softmax of a row is a lane's own work and one exchange with lane ^ 32, and the probabilities
// are the B operand of O^T = V^T P^T as they stand, the contraction's order being free as long as both operands agree on it.
// One pass over the keys with a running maximum and sum (fp32); the accumulators are rescaled only where a maximum rises by more
// than 2^8.  bf16: the probabilities, unnormalised and at most 2^8, are rounded to bf16 for the second product (relative 2^-9
// each, averaging over the keys), the sum is that of the unrounded ones.
//
// Where a batch has too few row tiles for the device the keys of a tile are cut into equal parts, each leaving its
// unnormalised output, maximum and sum, which a second kernel joins in a fixed order.
#include "respec_common.hpp"
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
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef s16x4 __attribute__((address_space(3))) *LdsTr;

constexpr float kRescaleSlack = 8.f;  // log2 units
constexpr int kMaxSplits = 16;
constexpr int kSplitGroups = 1024;    // work-groups up to which a call is split (bounds the workspace: 128 MiB of parts)

struct PromptParams {
    const char *q, *k, *v;
    char *out;
    float *lse;
    const int32_t *q_indptr;
    const int64_t *kv_indptr;                       // tokens back to back, or NULL:
    const int32_t *page_indptr, *page_table, *kv_len;  // pages
    int64_t ld_q, ld_k, ld_v;  // elements between tokens of q, k and v (pages: Hkv * D)
    int64_t total_kv;
    int32_t B, total_q, max_q, max_kv, num_pages, table_len, page_shift;
    int32_t Hq, Hkv, G;
    int32_t splits;          // parts of a tile's keys
    uint32_t g_mul, g_shift; // of a division by G (by_g)
    uint32_t q_and, q_xor;   // on the bits of q: a negative scale is taken out of it, a zero one makes it zero
    float scale2;            // |sm_scale| * log2(e)
    float *part_o;           // [tiles * Hkv * splits][rows][D]
    float *part_ml;          // [tiles * Hkv * splits][rows][2]
};

// x / G by a product: with s = ceil(log2 G) and g_mul = floor(2^32 (2^s - G) / G) + 1 this is exact for every x below 2^32.
__device__ inline int by_g(const PromptParams &p, int x) {
    const uint32_t t = __umulhi((uint32_t)x, p.g_mul);
    return p.G == 1 ? x : (int)((t + (((uint32_t)x - t) >> 1)) >> (p.g_shift - 1));
}

template <bool BF16, int D, int WAVES>
struct Shape {
    static constexpr int kThreads = WAVES * 64;
    static constexpr int kRows = WAVES * 32;              // packed rows of a work-group
    static constexpr int kSize = BF16 ? 2 : 4;
    static constexpr int kKeys = BF16 ? 64 : 32;          // of a tile
    static constexpr int kBlocks = kKeys / 32;            // of 32 keys
    static constexpr int kRowBytes = D * kSize;
    static constexpr int kChunks = kRowBytes / 16;        // 16-byte pieces of a key's row
    static constexpr int kTileBytes = kKeys * kRowBytes;
    static constexpr int kLoads = kKeys * kChunks / kThreads;  // pieces of K (and of V) that a thread moves per tile
    static constexpr int kWaveKeys = 64 / kChunks;        // keys that a wave moves with one load of every lane
    static constexpr int kDTiles = D / 32;
    static constexpr int kRing = WAVES == 8 ? 4 : 2;      // tiles of K and of V in LDS
    static constexpr int kLdsBytes = 2 * kRing * kTileBytes + 16;
    static_assert(kKeys * kChunks % kThreads == 0, "whole pieces per thread");
    static_assert(16 % kWaveKeys == 0, "a wave's load lies in one page");
};

// Where a 16-byte piece of a key's row lies in the row, so that the lanes that read together meet different banks: K is read as
// one piece per key (sixteen keys at a time), V (bf16) as four keys by 64 bytes, V (fp32) along a row.
template <bool BF16, int D>
__device__ inline int k_piece(int key, int c) {
    constexpr int kChunks = D * (BF16 ? 2 : 4) / 16;
    if constexpr (kChunks == 8) return c ^ ((key >> 1) & 7);
    else return c ^ (key & 15);  // (32 pieces: within each half of the row)
}
template <bool BF16, int D>
__device__ inline int v_piece(int key, int c) {
    if constexpr (!BF16) return c;
    else if constexpr (D == 128) return c ^ ((key & 3) << 2);
    else return c ^ (((key >> 1) & 1) << 2);
}

// Results of an operation on a lane's value and that of lane ^ 32.
__device__ inline float max_of_halves(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float sum_of_halves(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// What a work-group computes: a tile of packed rows of one KV head, and a part of the keys that it sees.
struct Job {
    Tile tile;
    int head, number;      // KV head; the work-group's place among the parts
    int64_t kv0;           // the sequence's first token (pages: its first entry of page_table)
    int L;                 // its tokens
    int row0, n_rows;      // first packed row of the tile, packed rows of the sequence
    int t_begin, t_end;    // tiles of keys
    int all;               // keys that all rows of the work-group see
};

// Tokens of sequence b and where they begin, inside the buffers whatever the arrays hold.
template <bool PAGED>
__device__ inline int length_of(const PromptParams &p, int b, int64_t &kv0) {
    if constexpr (PAGED) {
        kv0 = max(0, min(p.page_indptr[b], p.table_len));
        const int64_t pages = max((int64_t)0, (int64_t)min(p.page_indptr[b + 1], p.table_len) - kv0);
        return (int)max((int64_t)0, min(min((int64_t)p.kv_len[b], pages << p.page_shift), (int64_t)p.max_kv));
    } else {
        kv0 = max((int64_t)0, min(p.kv_indptr[b], p.total_kv));
        return (int)max((int64_t)0, min(min(p.kv_indptr[b + 1], p.total_kv) - kv0, (int64_t)p.max_kv));
    }
}

__device__ inline int bits_before(uint64_t mask) {  // set bits of lanes before this one
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// The number-th tile of a batch of up to 64 sequences (one per lane), those that see most keys first, in steps of kOrderStep keys:
// work-groups are given out in order, and a long one among the last would be waited for.  How many tiles see x keys or more is known
// for every sequence without looking at its tiles, so the step is found by bisection.  (16 packed prompts of 65 to 2,048 tokens at
// 28/4 heads take 140 us, in the order of the sequences 160; 8 chunks behind up to 8,192 tokens at 40/8 heads with their append 332,
// and 348; in steps of 64 keys no different.)
constexpr int kOrderStep = 256, kInTurn = 32;
template <bool PAGED, int ROWS>
__device__ inline bool find_longest(const PromptParams &p, int number, Tile &out, int &tokens, int64_t &first) {
    const int lane = threadIdx.x & 63;
    int q0 = 0, R = 0, L = 0;
    int64_t kv0 = 0;
    if (lane < p.B) {
        q0 = max(0, min(p.q_indptr[lane], p.total_q));
        R = max(0, min(min(p.q_indptr[lane + 1], p.total_q) - q0, p.max_q));
        L = length_of<PAGED>(p, lane, kv0);
    }
    const int tiles = (R * p.G + ROWS - 1) / ROWS, before = L - R;  // (before: negative where the first rows see nothing)
    auto reach = [&](int x) __attribute__((always_inline)) {  // this sequence's tiles that see kOrderStep x keys or more
        if (x <= 0) return tiles;
        if ((int64_t)x * kOrderStep > L || tiles == 0) return 0;
        const int first = ((max(x * kOrderStep - before - 1, 0) * p.G + 1) + ROWS - 1) / ROWS - 1;  // (the last tile's last row sees L keys)
        return tiles - max(0, min(first, tiles - 1));
    };
    auto all = [&](int x) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(wave_scan_add(reach(x)), 63); };
    if (number >= all(0)) return false;
    int x = 0, over = p.max_kv / kOrderStep + 1, n_over = 0;  // all(x) > number >= all(over)
    while (p.B > 1 && over - x > 1) {
        const int at = (x + over) / 2, n_at = all(at);
        if (n_at > number) x = at;
        else over = at, n_over = n_at;
    }
    const int more = p.B == 1 ? 0 : reach(over), mine = p.B == 1 ? tiles : reach(x) - more;  // (one sequence: its tiles from the last)
    // Among the tiles of a step one of every sequence in turn: an XCD, which is given every eighth work-group, then meets fewer sequences' keys
    // at a time than with one sequence after the other (16 prompts of 1,024 tokens at 28/4 heads take 161 us, and 166).  Of many sequences
    // that is too much for its L2, and one comes after the other (64 of 256 tokens 82 us, in turn 84).
    int rest = number - (p.B == 1 ? 0 : n_over), turn = 0;
    uint64_t left = __ballot(mine > 0);
    int at;
    if (__popcll(left) > kInTurn || p.B == 1) {
        const int sum = wave_scan_add(mine);
        at = (int)__builtin_ctzll(__ballot(sum > rest));
        turn = rest - __builtin_amdgcn_readlane(sum - mine, at);
    } else {
        for (int n = (int)__popcll(left); rest >= n; n = (int)__popcll(left)) {
            rest -= n;
            left = __ballot(mine > ++turn);
        }
        at = (int)__builtin_ctzll(__ballot((left >> lane & 1) != 0 && bits_before(left) == rest));
    }
    out.b = at;
    out.tiles = __builtin_amdgcn_readlane(tiles, at);
    out.index = __builtin_amdgcn_readlane(tiles - more, at) - 1 - turn;
    out.R = __builtin_amdgcn_readlane(R, at);
    out.q0 = __builtin_amdgcn_readlane(q0, at);
    tokens = __builtin_amdgcn_readlane(L, at);
    first = (int64_t)__builtin_amdgcn_readlane((int)(kv0 >> 32), at) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)kv0, at);
    return true;
}

// The number-th tile of row tiles, with its sequence's tokens and where they begin.  Batches of more than 64 sequences: one sequence after the
// other, each from the tile that sees most.
template <bool PAGED, int ROWS>
__device__ inline bool find_rows(const PromptParams &p, int number, Tile &out, int &tokens, int64_t &first) {
    if (p.B <= 64) return find_longest<PAGED, ROWS>(p, number, out, tokens, first);
    if (!find_tile(p.q_indptr, p.B, p.total_q, p.max_q, p.G, ROWS, number, out)) return false;
    out.index = out.tiles - 1 - out.index;  // (the longest of a sequence first)
    tokens = __builtin_amdgcn_readfirstlane(length_of<PAGED>(p, out.b, first));
    return true;
}

template <bool BF16, int D, int WAVES, bool PAGED>
__device__ inline bool find_job(const PromptParams &p, Job &j) {
    using S = Shape<BF16, D, WAVES>;
    j.head = blockIdx.x % p.Hkv;
    const int rest = blockIdx.x / p.Hkv, number = p.splits == 1 ? rest : rest / p.splits, split = rest - number * p.splits;
    j.number = blockIdx.x;
    if (!find_rows<PAGED, S::kRows>(p, number, j.tile, j.L, j.kv0)) return false;
    j.n_rows = j.tile.R * p.G;
    j.row0 = j.tile.index * S::kRows;
    const int last = min(j.row0 + S::kRows, j.n_rows) - 1;
    const int end = j.L - j.tile.R + by_g(p, last) + 1;  // the work-group's last row sees most
    const int tiles = max(0, (end + S::kKeys - 1) / S::kKeys);
    j.t_begin = p.splits == 1 ? 0 : tiles * split / p.splits;  // (at most 2^25 tiles, kMaxSplits parts)
    j.t_end = p.splits == 1 ? tiles : tiles * (split + 1) / p.splits;
    j.all = j.L - j.tile.R + by_g(p, j.row0) + 1;
    return true;
}

// This lane's row (columns lane % 32 of its wave's tile): it sees keys 0 .. lim-1.
struct RowOf {
    bool exists;
    int lim, head;
    int64_t token;
    int wave_sees, wave_all;  // keys that some row of the wave sees, that all of them see
};
__device__ inline RowOf row_of(const PromptParams &p, const Job &j, int wave, int col) {
    RowOf r;
    const int packed = j.row0 + wave * 32 + col, clamped = min(packed, j.n_rows - 1);
    r.exists = packed < j.n_rows;
    const int i = by_g(p, clamped);
    r.lim = j.L - j.tile.R + i + 1;
    r.head = j.head * p.G + clamped - i * p.G;
    r.token = j.tile.q0 + i;
    r.wave_sees = __builtin_amdgcn_readlane(r.lim, 31);
    r.wave_all = __builtin_amdgcn_readlane(r.lim, 0);
    return r;
}

// Q^T as the B operand: a lane's column is its row, its contraction slots the pieces 2x + half of the row.
template <int CHUNKS>
__device__ inline void load_q(const PromptParams &p, const RowOf &r, int D, int size, int half, u32x4 (&qf)[CHUNKS / 2]) {
    const char *qp = p.q + (r.token * p.ld_q + (int64_t)r.head * D) * size + half * 16;
#pragma unroll
    for (int x = 0; x < CHUNKS / 2; ++x) qf[x] = *reinterpret_cast<const u32x4 *>(qp + x * 32);
}
template <int N>
__device__ inline void sign_q(const PromptParams &p, u32x4 (&qf)[N]) {  // (apart: the loads are not waited for before others are requested)
#pragma unroll
    for (int x = 0; x < N; ++x)
        for (int w = 0; w < 4; ++w) qf[x][w] = (qf[x][w] & p.q_and) ^ p.q_xor;
}

typedef const __attribute__((address_space(4))) int32_t *ConstInts;  // (read through the scalar cache; nothing writes it meanwhile)

// Moves K or V pieces from global memory into registers and on into LDS: key wave * kWaveKeys + lane / kChunks + i * (keys of all
// waves) of a tile, piece lane % kChunks.  The keys of a wave's load lie in one page, so what differs between lanes is a 32-bit offset.
// Keys past the end are the last one's (they are never seen).
template <bool BF16, int D, int WAVES, bool PAGED>
struct Mover {
    using S = Shape<BF16, D, WAVES>;
    static constexpr int kSpots = PAGED ? S::kLoads : 1;
    struct Spot {             // where a tile lies, the same in K and V (all uniform)
        int64_t row[kSpots];  // of its first key, or of each load's
        int left[kSpots];     // keys behind that one
    };
    const char *k, *v;
    int wave, my_key;
    uint32_t my_piece;
    int L;
    int64_t kv0, ld_k, ld_v;  // (bytes)
    ConstInts table;
    int num_pages, shift;
    __device__ Mover(const PromptParams &p, const Job &j, int w, int lane) {
        wave = w;
        my_key = lane / S::kChunks;
        my_piece = (uint32_t)(lane % S::kChunks) * 16;
        k = p.k + (int64_t)j.head * S::kRowBytes;
        v = p.v + (int64_t)j.head * S::kRowBytes;
        L = j.L;
        kv0 = j.kv0;
        ld_k = p.ld_k * S::kSize;
        ld_v = p.ld_v * S::kSize;
        if constexpr (PAGED) {
            table = (ConstInts)(p.page_table + j.kv0);
            num_pages = p.num_pages;
            shift = p.page_shift;
        }
    }
    __device__ Spot find(int t) const {  // (a tile that begins within the sequence)
        Spot s;
#pragma unroll
        for (int i = 0; i < kSpots; ++i) {
            if constexpr (PAGED) {
                const int n = min(t * S::kKeys + i * (WAVES * S::kWaveKeys) + wave * S::kWaveKeys, L - 1);
                const int64_t page = max(0, min(table[n >> shift], num_pages - 1));
                s.row[i] = (page << shift) + (n & ((1 << shift) - 1));
                s.left[i] = L - 1 - n;
            } else {
                s.row[i] = kv0 + (int64_t)t * S::kKeys;
                s.left[i] = L - 1 - t * S::kKeys;
            }
        }
        return s;
    }
    template <bool V>
    __device__ void load(const Spot &s, u32x4 (&x)[S::kLoads]) const {
        const int64_t ld = V ? ld_v : ld_k;
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i) {
            const int at = PAGED ? i : 0, mine = PAGED ? my_key : key(i);
            const uint32_t off = __umul24((uint32_t)min(mine, s.left[at]), (uint32_t)ld) + my_piece;
            x[i] = *reinterpret_cast<const u32x4 *>((V ? v : k) + s.row[at] * ld + off);
        }
    }
    __device__ int key(int i) const { return i * (WAVES * S::kWaveKeys) + wave * S::kWaveKeys + my_key; }
    __device__ void put_k(char *tile, const u32x4 (&x)[S::kLoads]) const {
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i)
            *reinterpret_cast<u32x4 *>(tile + key(i) * S::kRowBytes + k_piece<BF16, D>(key(i), my_piece / 16) * 16) = x[i];
    }
    // `masked`: some row of the work-group does not see all of the tile.  A product would carry a value that is not finite to it all the
    // same: such values count as zero here and reach the rows that see them at the end.
    __device__ void put_v(char *tile, u32x4 (&x)[S::kLoads], bool masked, int *not_finite) const {
        if (masked) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < S::kLoads; ++i)
                for (int w = 0; w < 4; ++w) {
                    const bool hi = (x[i][w] & 0x7f800000u) == 0x7f800000u, lo = BF16 && (x[i][w] & 0x7f80u) == 0x7f80u;
                    bad |= hi || lo;
                    x[i][w] &= (hi ? (BF16 ? 0xffffu : 0u) : ~0u) & (lo ? 0xffff0000u : ~0u);
                }
            if (bad) *not_finite = 1;
        }
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i)
            *reinterpret_cast<u32x4 *>(tile + key(i) * S::kRowBytes + v_piece<BF16, D>(key(i), my_piece / 16) * 16) = x[i];
    }
};

// Writes a lane's row: O^T in accumulator tiles (d = 32 d-tile + 8 (x / 4) + 4 half + x % 4), its maximum (log2 units) and sum.
template <bool BF16, int D, int WAVES, bool PAGED>
__device__ inline void finish(const PromptParams &p, const Job &j, const RowOf &r, int wave, int half, int col, floatx16 (&o)[D / 32], float m, float l,
                              int not_finite, char *lds) {
    using S = Shape<BF16, D, WAVES>;
    const int64_t slot = (int64_t)j.number * S::kRows + wave * 32 + col;
    if (p.splits > 1) {
        if (r.exists && half == 0) *reinterpret_cast<floatx2 *>(p.part_ml + slot * 2) = floatx2{m, l};
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; x += 4)
                if (r.exists) *reinterpret_cast<floatx4 *>(p.part_o + slot * D + d * 32 + 2 * x + 4 * half) = floatx4{o[d][x], o[d][x + 1], o[d][x + 2], o[d][x + 3]};
    } else if constexpr (BF16) {
        // Through LDS, so that whole rows are written, sixteen bytes a lane: the wave's own 32 rows, pieces placed as K's are.  Past the caches,
        // which K and V fill (32 prompts of 512 tokens at 28/4 heads 104 us, with ordinary stores 111).
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;  // (no visible key: zero; NaN stays)
        char *const mine = lds + wave * 32 * S::kRowBytes;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; x += 4) {  // four d in a row
                const bf16x2 a = __builtin_convertvector(floatx2{o[d][x] * inv, o[d][x + 1] * inv}, bf16x2);
                const bf16x2 c = __builtin_convertvector(floatx2{o[d][x + 2] * inv, o[d][x + 3] * inv}, bf16x2);
                *reinterpret_cast<u32x2 *>(mine + col * S::kRowBytes + k_piece<true, D>(col, d * 4 + x / 4) * 16 + 8 * half) =
                    u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c)};
            }
        if (p.lse && half == 0 && r.exists) p.lse[r.token * p.Hq + r.head] = l == 0.f ? -INFINITY : m * 0.693147180559945309f + logf(l);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const int lane = half * 32 + col, piece = lane % S::kChunks;
#pragma unroll
        for (int i = 0; i < 32 / S::kWaveKeys; ++i) {
            const int at = i * S::kWaveKeys + lane / S::kChunks, packed = j.row0 + wave * 32 + at;
            const u32x4 x = *reinterpret_cast<const u32x4 *>(mine + at * S::kRowBytes + k_piece<true, D>(at, piece) * 16);
            if (packed < j.n_rows) {
                const int row = by_g(p, packed);
                char *const to = p.out + ((j.tile.q0 + row) * p.Hq + j.head * p.G + packed - row * p.G) * (int64_t)S::kRowBytes + piece * 16;
                __builtin_nontemporal_store(x, reinterpret_cast<u32x4 *>(to));
            }
        }
    } else if (r.exists) {
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
        char *op = p.out + (r.token * p.Hq + r.head) * (int64_t)S::kRowBytes;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; x += 4)
                *reinterpret_cast<floatx4 *>(op + (d * 32 + 2 * x + 4 * half) * 4) =
                    floatx4{o[d][x] * inv, o[d][x + 1] * inv, o[d][x + 2] * inv, o[d][x + 3] * inv};
        if (p.lse && half == 0) p.lse[r.token * p.Hq + r.head] = l == 0.f ? -INFINITY : m * 0.693147180559945309f + logf(l);
    }
    if (not_finite == 0) return;  // (uniform)
    // The values that put_v left out, added to what the work-group (WAVES = 1: the wave) has written: a row and a d of it per thread.
    if constexpr (WAVES > 1) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        __builtin_amdgcn_wave_barrier();
    }
    const int first_key = max(j.t_begin, j.all / S::kKeys) * S::kKeys, end_key = j.t_end * S::kKeys;
    for (int e = threadIdx.x; e < S::kRows * D; e += S::kThreads) {
        const int row = j.row0 + e / D, d = e % D;
        if (row >= j.n_rows) break;
        const int sees = min(end_key, j.L - j.tile.R + by_g(p, row) + 1);
        float sum = 0.f;
        for (int n = first_key; n < sees; ++n) {
            int64_t at = j.kv0 + n;
            if constexpr (PAGED)
                at = ((int64_t)max(0, min(p.page_table[j.kv0 + (n >> p.page_shift)], p.num_pages - 1)) << p.page_shift) + (n & ((1 << p.page_shift) - 1));
            const char *vp = p.v + (at * p.ld_v + (int64_t)j.head * D + d) * S::kSize;
            const float x = BF16 ? __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(vp) << 16) : *reinterpret_cast<const float *>(vp);
            if (!(fabsf(x) < INFINITY)) sum += x;
        }
        if (sum == 0.f) continue;  // (nothing but +-inf or NaN is added)
        if (p.splits > 1) {
            p.part_o[((int64_t)j.number * S::kRows + e / D) * D + d] += sum;
        } else {
            char *op = p.out + (((j.tile.q0 + by_g(p, row)) * p.Hq + j.head * p.G + row - by_g(p, row) * p.G) * (int64_t)D + d) * S::kSize;
            if constexpr (BF16) {
                const float x = __uint_as_float((uint32_t)*reinterpret_cast<uint16_t *>(op) << 16) + sum;
                *reinterpret_cast<uint16_t *>(op) = __builtin_bit_cast(uint16_t, (__bf16)x);
            } else {
                *reinterpret_cast<float *>(op) += sum;
            }
        }
    }
}

// Score x of a block of 32 keys is key 8 (x / 4) + 4 half + x % 4.
__device__ inline void mask_scores(floatx16 &s, int first_key, int half, int lim) {
#pragma unroll
    for (int x = 0; x < 16; ++x)
        if (first_key + 8 * (x / 4) + 4 * half + x % 4 >= lim) s[x] = -INFINITY;
}

// fp32: one tile of 32 keys after the other.  WAVES = 4: four waves of 32 rows each read the same tiles, two of K and two of V in
// LDS.  WAVES = 1: the four waves of a work-group hold the same 32 rows, each takes every fourth tile, through LDS of its own
// and without a barrier, and the first one joins what they found.  Large calls are bound by the fp32 matrix rate (64 keys of 128 rows
// take a compute unit 8.4 us at D = 128), small ones by latency: 4 prompts of up to 200 tokens at 4/1 heads of 64 take 10.7 us, of which
// two tiles of keys 4.
template <int D, int WAVES, bool PAGED>
__global__ __launch_bounds__(256, WAVES == 4 ? 2 : 1) void prompt_f32_kernel(PromptParams p) {
    using S = Shape<false, D, WAVES>;
    constexpr bool kShared = WAVES == 4;
    constexpr int kStride = kShared ? 1 : 4;
    extern __shared__ __align__(16) char lds[];
    __shared__ int sh_not_finite;
    Job job;
    if (!find_job<false, D, WAVES, PAGED>(p, job)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    char *const lds_k = kShared ? lds : lds + wave * 2 * S::kTileBytes, *const lds_v = lds_k + (kShared ? 2 : 1) * S::kTileBytes;
    const RowOf row = row_of(p, job, kShared ? wave : 0, col);
    u32x4 qf[S::kChunks / 2];
    load_q<S::kChunks>(p, row, D, S::kSize, half, qf);
    const Mover<false, D, WAVES, PAGED> mover(p, job, kShared ? wave : 0, lane);
    if (threadIdx.x == 0) sh_not_finite = 0;
    auto ready = [&]() __attribute__((always_inline)) {  // (what was put is there to read)
        if constexpr (kShared) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };

    floatx16 o[S::kDTiles];
#pragma unroll
    for (int d = 0; d < S::kDTiles; ++d)
        for (int x = 0; x < 16; ++x) o[d][x] = 0.f;
    float m = -INFINITY, l = 0.f;
    u32x4 kr[S::kLoads], vr[S::kLoads];
    auto put = [&](int buffer, int t) __attribute__((always_inline)) {
        mover.put_k(lds_k + buffer * S::kTileBytes, kr);
        mover.put_v(lds_v + buffer * S::kTileBytes, vr, (t + 1) * S::kKeys > job.all, &sh_not_finite);
    };
    const int first = job.t_begin + (kShared ? 0 : wave);
    if (first < job.t_end) {  // (uniform in the waves that share a tile)
        const auto spot = mover.find(first);
        mover.template load<false>(spot, kr);
        mover.template load<true>(spot, vr);
    }
    sign_q(p, qf);
    __syncthreads();  // (sh_not_finite)
    if (first < job.t_end) {
        put(0, first);
        ready();
    }
    for (int t = first; t < job.t_end; t += kStride) {
        const int buffer = kShared ? (t - first) & 1 : 0;
        if (t + kStride < job.t_end) {
            const auto spot = mover.find(t + kStride);
            mover.template load<false>(spot, kr);
            mover.template load<true>(spot, vr);
        }
        if (t * S::kKeys < row.wave_sees) {
            const char *kb = lds_k + buffer * S::kTileBytes, *vb = lds_v + buffer * S::kTileBytes;
            floatx16 s;
            for (int x = 0; x < 16; ++x) s[x] = 0.f;
#pragma unroll
            for (int x = 0; x < S::kChunks / 2; ++x) {
                const u32x4 a = *reinterpret_cast<const u32x4 *>(kb + col * S::kRowBytes + k_piece<false, D>(col, 2 * x + half) * 16);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[y]), __uint_as_float(qf[x][y]), s, 0, 0, 0);
            }
            if ((t + 1) * S::kKeys > row.wave_all) mask_scores(s, t * S::kKeys, half, row.lim);
            float top = s[0];
#pragma unroll
            for (int x = 1; x < 16; ++x) top = fmaxf(top, s[x]);
            top = max_of_halves(top) * p.scale2;
            if (__ballot(top > m + kRescaleSlack) != 0) {  // (m = -inf: any finite score)
                const float m_new = top > m + kRescaleSlack ? top : m;
                const float f = m == m_new ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
                m = m_new;
                l *= f;
#pragma unroll
                for (int d = 0; d < S::kDTiles; ++d)
                    for (int x = 0; x < 16; ++x) o[d][x] *= f;
            }
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                s[x] = __builtin_amdgcn_exp2f(fmaf(s[x], p.scale2, -ref));
                l += s[x];
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const int key = 8 * (x / 4) + 4 * half + x % 4;
#pragma unroll
                for (int d = 0; d < S::kDTiles; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float *>(vb + key * S::kRowBytes + (d * 32 + col) * 4), s[x], o[d],
                                                                0, 0, 0);
            }
        }
        if constexpr (!kShared) ready();  // (the tile has been read)
        if (t + kStride < job.t_end) put(kShared ? buffer ^ 1 : 0, t + kStride);
        ready();
    }
    l = sum_of_halves(l);
    if constexpr (!kShared) {
        constexpr int kPieces = S::kDTiles * 4;  // of a lane's accumulators
        static_assert(kPieces * 1024 == S::kTileBytes, "a wave's accumulators fill its tile of K");
        if (wave != 0) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                *reinterpret_cast<floatx4 *>(lds_k + i * 1024 + lane * 16) =
                    floatx4{o[i / 4][i % 4 * 4], o[i / 4][i % 4 * 4 + 1], o[i / 4][i % 4 * 4 + 2], o[i / 4][i % 4 * 4 + 3]};
            *reinterpret_cast<floatx2 *>(lds_v + lane * 8) = floatx2{m, l};
        }
        __syncthreads();
        if (wave != 0) return;
        floatx2 ml[4] = {{m, l}};
        float most = m;
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            ml[w] = *reinterpret_cast<const floatx2 *>(lds_v + w * 2 * S::kTileBytes + lane * 8);
            most = fmaxf(most, ml[w][0]);
        }
        l = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = ml[w][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[w][0] - most);  // (a NaN of l or o stays one)
            l = fmaf(ml[w][1], f, l);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                if (w == 0) {
                    for (int x = 0; x < 4; ++x) o[i / 4][i % 4 * 4 + x] *= f;
                    continue;
                }
                const floatx4 other = *reinterpret_cast<const floatx4 *>(lds_k + w * 2 * S::kTileBytes + i * 1024 + lane * 16);
                for (int x = 0; x < 4; ++x) o[i / 4][i % 4 * 4 + x] = fmaf(other[x], f, o[i / 4][i % 4 * 4 + x]);
            }
        }
        m = most;
    }
    finish<false, D, WAVES, PAGED>(p, job, row, kShared ? wave : 0, half, col, o, m, l, sh_not_finite, lds);
}

// f(0), f(1) ... f(N-1), each with its number as a type.
template <int N, typename F, int... I>
__device__ __attribute__((always_inline)) inline void each_of(F &&f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __attribute__((always_inline)) inline void each(F &&f) {
    each_of<N>(f, std::make_integer_sequence<int, N>{});
}

// bf16: the scores of tile t+1 are multiplied while the exponentials of tile t are computed; step t reads K of t+1 and V of t.
// Eight waves: LDS holds four tiles of K and four of V (128 KiB at D = 128, one work-group per compute unit), step t fetches K of t+3
// and V of t+2; what a step writes is read two steps later and what it writes over was read two steps before, so one barrier
// for two steps is enough.  Four waves: two tiles of each and two work-groups per compute unit, K of t+2 and V of t+1, a
// barrier per step.  The loop is written for as many steps as there are tiles in
// LDS, so that a tile's place is a constant.
// One prompt of 16,384 tokens at 16/2 heads of 128 takes 970 to 1,020 us by the card (1.1 PFLOP/s): the matrix pipes are busy 59 % of the cycles, of a clock
// that the power holds at 1.7 GHz.  16 prompts of 65 to 2,048 at 28/4 heads take 140 us: a work-group spends 14,000 of its 44,000
// cycles on its rows, Q, the first keys and the output, half of it behind the other work-group of its compute unit.
template <int D, int WAVES, bool PAGED>
__global__ __launch_bounds__(WAVES * 64, 2) void prompt_bf16_kernel(PromptParams p) {
    using S = Shape<true, D, WAVES>;
    constexpr int kRing = S::kRing, kFetch = kRing == 4 ? 3 : 2;  // K is fetched so many tiles ahead, V one less
    extern __shared__ __align__(16) char lds[];  // kRing tiles of K, kRing of V, and a word
    int &sh_not_finite = *reinterpret_cast<int *>(lds + 2 * kRing * S::kTileBytes);
    Job job;
    if (!find_job<true, D, WAVES, PAGED>(p, job)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    const Mover<true, D, WAVES, PAGED> mover(p, job, wave, lane);
    typedef typename Mover<true, D, WAVES, PAGED>::Spot Spot;
    Spot spot{};  // of the tile whose V the next step fetches
    u32x4 kr[kFetch][S::kLoads], vr[kFetch - 1][S::kLoads];
    const int tiles = job.t_end - job.t_begin;
#pragma unroll
    for (int i = 0; i < kFetch; ++i)
        if (i < tiles) {
            spot = mover.find(job.t_begin + i);
            mover.template load<false>(spot, kr[i]);
            if (i < kFetch - 1) mover.template load<true>(spot, vr[i < kFetch - 1 ? i : 0]);
        }
    const RowOf row = row_of(p, job, wave, col);
    u32x4 qf[S::kChunks / 2];
    load_q<S::kChunks>(p, row, D, S::kSize, half, qf);
    if (threadIdx.x == 0) sh_not_finite = 0;
    __syncthreads();

    // Where this lane reads: a key's pieces of K; for V the transposing read's sixteen lanes address four keys by sixteen d and
    // receive one d of the four keys each.  The place of a piece within its row is an exclusive or, so the x-th piece pair of K lies at
    // k_at ^ 32 x and the d-th tile of V at v_at ^ 64 d.
    int k_at = col * S::kRowBytes + k_piece<true, D>(col, half) * 16;
    const int i16 = lane & 15, v_key = half * 4 + (i16 >> 2), d0 = ((lane & 16) + 4 * (i16 & 3)) * 2;
    int v_at = kRing * S::kTileBytes + v_key * S::kRowBytes + v_piece<true, D>(v_key, d0 >> 4) * 16 + (d0 & 15);

    floatx16 o[S::kDTiles];
#pragma unroll
    for (int d = 0; d < S::kDTiles; ++d)
        for (int x = 0; x < 16; ++x) o[d][x] = 0.f;
    float m = -INFINITY, ref = 0.f, l = 0.f;
    floatx16 s_even[S::kBlocks], s_odd[S::kBlocks];

    auto largest = [&](const floatx16(&s)[S::kBlocks]) __attribute__((always_inline)) {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
            for (int x = b == 0; x < 16; ++x) top = fmaxf(top, s[b][x]);
        return top;
    };
    auto mask = [&](int t, floatx16(&s)[S::kBlocks]) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b) mask_scores(s[b], t * S::kKeys + b * 32, half, row.lim);
    };
    auto rescale = [&](float top) __attribute__((always_inline)) {  // with the largest score that this lane has
        top = max_of_halves(top) * p.scale2;
        if (__ballot(top > m + kRescaleSlack) == 0) return;  // (m = -inf: any finite score)
        const float m_new = top > m + kRescaleSlack ? top : m;
        const float f = m == m_new ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        ref = m == -INFINITY ? 0.f : m;
        l *= f;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
            for (int x = 0; x < 16; ++x) o[d][x] *= f;
    };
    // Two probabilities of sixteen keys' B operand, the n-th pair of all: slot j is key 8 (j / 4) + 4 half + j % 4 of them.
    auto pair = [&](auto n_, const floatx16(&s)[S::kBlocks], u32x4(&pf)[2 * S::kBlocks]) __attribute__((always_inline)) {
        constexpr int n = decltype(n_)::value, g = n / 4, j = n % 4 * 2;
        const float a = __builtin_amdgcn_exp2f(fmaf(s[g / 2][g % 2 * 8 + j], p.scale2, -ref));
        const float c = __builtin_amdgcn_exp2f(fmaf(s[g / 2][g % 2 * 8 + j + 1], p.scale2, -ref));
        l += a;
        l += c;
        asm volatile("" : "+v"(l));  // (added now: later, the sixteen pairs would have to be kept)
        pf[g][j / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, c}, bf16x2));
    };
    auto read_v = [&](int g, int d, int tile) __attribute__((always_inline)) {
        s16x4 vt[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) vt[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTr)(lds + (v_at ^ (64 * d)) + (tile + (g * 16 + j * 8) * S::kRowBytes)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(vt[0], vt[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // Step t (not the last), the tile's scores in s with their maximum taken into account; `place`: (t - t_begin) % kRing.
    // Written in the order it is to run in: a product, an LDS read kAhead products before its use, and a share of the rest.
    auto step = [&](auto place, int t, floatx16(&s)[S::kBlocks], floatx16(&next)[S::kBlocks]) __attribute__((always_inline)) {
        constexpr int kPlace = decltype(place)::value;
        constexpr int kFirst = S::kBlocks * S::kChunks / 2, kSecond = 2 * S::kBlocks * S::kDTiles, kAhead = 4;
        constexpr int kPairs = 16 * S::kBlocks / 2, kEarly = kPairs * 5 / 8;  // pairs of probabilities; those along with the first products
        u32x4 moved[S::kLoads];  // K in the first half of the step, V in the second
        const Spot after = mover.find(min(t + kFetch, job.t_end - 1));
        mover.template load<false>(after, moved);
        if constexpr (WAVES == 4) asm volatile("" : "+v"(k_at), "+v"(v_at));  // (twelve addresses that do not change would not fit beside 16 pieces)
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 ahead[kAhead];
        u32x4 pf[2 * S::kBlocks];
        auto read = [&](auto i_) __attribute__((always_inline)) {
            constexpr int i = decltype(i_)::value;
            if constexpr (i < kFirst) {
                constexpr int b = i % S::kBlocks, x = i / S::kBlocks;
                ahead[i % kAhead] = *reinterpret_cast<const bf16x8 *>(lds + (k_at ^ (32 * x)) + ((kPlace + 1) % kRing * S::kTileBytes + b * 32 * S::kRowBytes));
            } else if constexpr (i < kFirst + kSecond) {
                ahead[i % kAhead] = read_v((i - kFirst) / S::kDTiles, (i - kFirst) % S::kDTiles, kPlace % kRing * S::kTileBytes);
            }
        };
        float top = -INFINITY;
        each<kAhead>([&](auto i) __attribute__((always_inline)) { read(i); });
        __builtin_amdgcn_sched_barrier(0);
        each<kFirst + kSecond>([&](auto i_) __attribute__((always_inline)) {
            constexpr int i = decltype(i_)::value;
            if constexpr (i == kFirst) {  // (past the last tile: not read)
                mover.put_k(lds + (kPlace + kFetch) % kRing * S::kTileBytes, moved);
                mover.template load<true>(spot, moved);
                spot = after;
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (i < kFirst) {
                constexpr int b = i % S::kBlocks, x = i / S::kBlocks;
                const floatx16 none{};
                next[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[i % kAhead], __builtin_bit_cast(bf16x8, qf[x]), x == 0 ? none : next[b], 0, 0, 0);
            } else {
                constexpr int g = (i - kFirst) / S::kDTiles, d = (i - kFirst) % S::kDTiles;
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[i % kAhead], __builtin_bit_cast(bf16x8, pf[g]), o[d], 0, 0, 0);
            }
            read(std::integral_constant<int, i + kAhead>{});
            if constexpr (i < kFirst) {
                constexpr int from = i * kEarly / kFirst, to = (i + 1) * kEarly / kFirst;
                each<to - from>([&](auto n) __attribute__((always_inline)) { pair(std::integral_constant<int, from + decltype(n)::value>{}, s, pf); });
            } else {  // the other pairs, none later than the products before its own, then the maximum
                constexpr int n = kEarly + i - kFirst, k = i - kFirst - (kPairs - kEarly), kRest = kSecond - (kPairs - kEarly);
                if constexpr (n < kPairs) pair(std::integral_constant<int, n>{}, s, pf);
                else
#pragma unroll
                    for (int x = 16 * S::kBlocks * k / kRest; x < 16 * S::kBlocks * (k + 1) / kRest; ++x) top = fmaxf(top, next[x / 16][x % 16]);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        if ((t + 2) * S::kKeys > row.wave_all) {  // (uniform)
            mask(t + 1, next);
            top = largest(next);
        }
        rescale(top);
        mover.put_v(lds + (kRing + (kPlace + kFetch - 1) % kRing) * S::kTileBytes, moved, (t + kFetch) * S::kKeys > job.all, &sh_not_finite);
        if constexpr (kRing == 2 || kPlace % 2 == 1) __syncthreads();
    };

    if (job.t_begin < job.t_end) {  // (uniform)
        int t = job.t_begin;
#pragma unroll
        for (int i = 0; i < kFetch; ++i)
            if (i < tiles) mover.put_k(lds + i * S::kTileBytes, kr[i]);
#pragma unroll
        for (int i = 0; i < kFetch - 1; ++i)
            if (i < tiles) mover.put_v(lds + (kRing + i) * S::kTileBytes, vr[i], (t + i + 1) * S::kKeys > job.all, &sh_not_finite);
        sign_q(p, qf);
        __syncthreads();
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
            for (int x = 0; x < S::kChunks / 2; ++x) {
                const bf16x8 a = *reinterpret_cast<const bf16x8 *>(lds + (k_at ^ (32 * x)) + b * 32 * S::kRowBytes);
                const floatx16 none{};
                s_even[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, qf[x]), x == 0 ? none : s_even[b], 0, 0, 0);
            }
        if ((t + 1) * S::kKeys > row.wave_all) mask(t, s_even);
        rescale(largest(s_even));
        __syncthreads();  // (the first tile's K is read by all before it is written over)
        int place = 0;  // of the last tile
        for (;;) {
            if (t + 1 >= job.t_end) break;
            step(std::integral_constant<int, 0>{}, t, s_even, s_odd);
            if (t + 2 >= job.t_end) {
                place = 1;
                break;
            }
            step(std::integral_constant<int, 1>{}, t + 1, s_odd, s_even);
            t += 2;
            if constexpr (kRing == 4) {
                if (t + 1 >= job.t_end) {
                    place = 2;
                    break;
                }
                step(std::integral_constant<int, 2>{}, t, s_even, s_odd);
                if (t + 2 >= job.t_end) {
                    place = 3;
                    break;
                }
                step(std::integral_constant<int, 3>{}, t + 1, s_odd, s_even);
                t += 2;
            }
        }
        if (place % 2 == 1)
            for (int b = 0; b < S::kBlocks; ++b) s_even[b] = s_odd[b];
        u32x4 pf[2 * S::kBlocks];
        each<16 * S::kBlocks / 2>([&](auto n) __attribute__((always_inline)) { pair(n, s_even, pf); });
#pragma unroll
        for (int g = 0; g < 2 * S::kBlocks; ++g)
#pragma unroll
            for (int d = 0; d < S::kDTiles; ++d)
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v(g, d, place * S::kTileBytes), __builtin_bit_cast(bf16x8, pf[g]), o[d], 0, 0, 0);
        __syncthreads();  // (sh_not_finite)
    }
    const int not_finite = sh_not_finite;
    int again = col;  // (the row's place is worked out again rather than kept)
    asm volatile("" : "+v"(again));
    finish<true, D, WAVES, PAGED>(p, job, row_of(p, job, wave, again), wave, half, again, o, m, sum_of_halves(l), not_finite, lds);
}

// Joins the parts of a tile's keys: a thread per packed row and four elements.  Bound by its launch and the parts' bytes (5.4 us and 3.6 TB/s
// with their writing).
template <bool BF16, int D, int ROWS, bool PAGED>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptParams p) {
    constexpr int kQuads = D / 4, kPerBlock = 256 / kQuads;  // rows of a work-group
    constexpr int kBlocks = ROWS / kPerBlock;                // work-groups of a tile
    const int piece = blockIdx.x % kBlocks, head = blockIdx.x / kBlocks % p.Hkv, number = blockIdx.x / kBlocks / p.Hkv;
    Tile tile;
    int tokens;
    int64_t first;
    if (!find_rows<PAGED, ROWS>(p, number, tile, tokens, first)) return;
    const int row = piece * kPerBlock + threadIdx.x / kQuads, quad = threadIdx.x % kQuads;
    const int packed = tile.index * ROWS + row;
    if (packed >= tile.R * p.G) return;
    float m = -INFINITY, l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < p.splits; ++s) {
        const int64_t slot = (((int64_t)number * p.splits + s) * p.Hkv + head) * ROWS + row;
        const floatx2 ml = *reinterpret_cast<const floatx2 *>(p.part_ml + slot * 2);
        if (ml[1] == 0.f) continue;  // (no key of this part is seen)
        const floatx4 x = *reinterpret_cast<const floatx4 *>(p.part_o + slot * D + quad * 4);
        const float m_new = fmaxf(m, ml[0]);
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new), e = __builtin_amdgcn_exp2f(ml[0] - m_new);
        l = l * f + ml[1] * e;
        for (int j = 0; j < 4; ++j) o[j] = o[j] * f + x[j] * e;
        m = m_new;
    }
    const int i_row = by_g(p, packed), q_head = head * p.G + packed - i_row * p.G;
    const int64_t at = (tile.q0 + i_row) * p.Hq + q_head;
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    for (int j = 0; j < 4; ++j) o[j] *= inv;
    if constexpr (BF16) {
        const bf16x2 a = __builtin_convertvector(floatx2{o[0], o[1]}, bf16x2), c = __builtin_convertvector(floatx2{o[2], o[3]}, bf16x2);
        *reinterpret_cast<u32x2 *>(p.out + (at * D + quad * 4) * 2) = u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c)};
    } else {
        *reinterpret_cast<floatx4 *>(p.out + (at * D + quad * 4) * 4) = o;
    }
    if (p.lse && quad == 0) p.lse[at] = l == 0.f ? -INFINITY : m * 0.693147180559945309f + logf(l);
}

// ------------------------------------------------------------------------------------------ host side
struct Plan {
    int64_t tiles;  // bound of the row tiles of a KV head
    int32_t waves, splits;
    size_t o_bytes, ws_bytes;
    size_t most_bytes;  // that a call with no larger sizes can need
};

struct PartBytes {
    size_t o, all;
};
PartBytes part_bytes(size_t slots, int32_t D) {
    const size_t o = round_up(slots * D * sizeof(float), 256);
    return {o, std::max<size_t>(256, o + round_up(slots * 2 * sizeof(float), 256))};
}

// How a call is run: the form (bf16: four waves, 128 packed rows, two work-groups on a compute unit; eight waves, 256 rows, one; fp32:
// 128 rows, or 32 whose tiles of keys four waves share out) and the parts its keys are cut into, whichever this estimate of the time in microseconds makes least.  A work-group costs `over`
// tiles of keys beside those that it sees; `step` is what a tile of 64 keys takes of a compute unit at D = 128, `lone` what it takes
// where no second work-group shares the unit.  The call takes the work of all groups over 256 units, or the longest group, and where
// the groups are alike (many keys before the chunk) whole rounds of them, of which half is counted for several sequences, as those
// are seldom of one length; parts cost a launch and their bytes.  The constants are fitted to 3,200 timings (1 to 64 prompts,
// chunks of 1 to 4,000 tokens behind 0 to 30,000, six head layouts, D 64 and 128, both forms, 1 to 16 parts): the form picked is on
// the mean 1.4 % behind the best of its shape.  8 chunks of 512 behind 7,680 at 40/8 heads: 660 us with eight waves, 701 with four.
// Eight waves at 28/4 heads of 128: 8 prompts of 2,048 take 258 us, with four 272; 64 of 128 take 46 us, with four 37.
// fp32 at 8/2 heads of 64: 4 prompts of 200 tokens take 12 us with four waves on 32 rows, 17 with 128; 32 of them 39 us, and 28.
// One chunk of 40 tokens behind 8,000: 30 us in 16 parts, 33 in 8; 512 behind 16,000, twice: 245 us in 2 parts, 306 in 3, 376 whole.
struct Cost {
    float step, lone, over, base;
};
constexpr Cost kFour{1.0f, 1.3f, 3.65f, 11.1f}, kEight{1.79f, 1.79f, 5.5f, 8.f}, kF32{7.5f, 10.6f, 0.25f, 7.9f}, kF32Keys{3.9f, 2.2f, 1.8f, 8.1f};

float estimate(const Cost &c, int32_t B, int64_t groups, int splits, int rows, float mean_q, int32_t max_q, int32_t max_kv, int32_t D, bool bf16) {
    const float before = (float)std::max(0, max_kv - max_q), alike = before / max_kv * (B == 1 ? 1.f : 0.5f);
    const float mean = (before + mean_q / 2) / 64 / splits + c.over, longest = max_kv / 64.f / splits + c.over;
    const int64_t up = (groups * splits + 255) / 256;
    const float odd = up % 2 == 1 ? c.lone - c.step : 0.f;
    const float even = groups * splits / 256.f * c.step * mean, whole = (up * c.step + odd) * mean;
    const float t = std::max(even + alike * (whole - even), longest * c.lone);
    const float parts = splits == 1 ? 0.f : 5.4f + groups * splits * (float)rows * D * 8 / 3.6e6f;
    return c.base + (D == 128 ? 1.f : bf16 ? 0.6f : 0.52f) * t + parts;
}

bool make_plan(int32_t B, int32_t total_q, int32_t max_q, int32_t max_kv, int32_t Hq, int32_t Hkv, int32_t D, respec_dtype_t dt, Plan &pl) {
    if (B <= 0 || total_q <= 0 || max_q <= 0 || max_kv <= 0 || Hq <= 0 || Hkv <= 0) return false;
    if (Hq % Hkv != 0 || (D != 64 && D != 128) || (dt != RESPEC_F32 && dt != RESPEC_BF16)) return false;
    const int32_t G = Hq / Hkv;
    if ((int64_t)std::min(max_q, total_q) * G >= (1 << 30)) return false;
    max_q = std::min(max_q, total_q);
    const Knobs kn = knobs();
    const long waves = kn.get(&Knobs::prompt_waves, 0), splits = kn.get(&Knobs::prompt_splits, 0);
    const float mean_q = std::min((float)max_q, (float)total_q / B);
    float least = INFINITY;
    size_t most = 0;  // slots: all that the rule below may cut a call into, whose sizes are no larger
    for (const int w : {8, 4, 1}) {
        const bool fits = dt == RESPEC_F32 ? w != 8 : w != 1, forced = dt == RESPEC_F32 ? waves == 1 || waves == 4 : waves == 4 || waves == 8;
        if (!fits || (forced && w != waves)) continue;
        const int64_t tiles = tiles_bound(B, total_q, max_q, G, w * 32), groups = tiles * Hkv;
        if (max_kv >= 128) most = std::max(most, (size_t)std::min<int64_t>(kSplitGroups, groups * std::min(kMaxSplits, max_kv / 64)) * w * 32);
        for (const int s : {1, 2, 3, 4, 6, 8, 12, kMaxSplits}) {
            if (s > 1 && (s > max_kv / 64 || groups * s > kSplitGroups)) break;
            const float t = estimate(dt == RESPEC_F32 ? (w == 4 ? kF32 : kF32Keys) : w == 8 ? kEight : kFour, B, groups, s, w * 32, mean_q, max_q, max_kv, D, dt == RESPEC_BF16);
            if (!(t < least)) continue;
            least = t;
            pl.waves = w;
            pl.splits = s;
            pl.tiles = tiles;
        }
    }
    if (splits >= 1 && splits <= kMaxSplits) pl.splits = (int32_t)splits;
    const size_t slots = pl.splits > 1 ? (size_t)(pl.tiles * Hkv) * pl.splits * pl.waves * 32 : 0;
    const PartBytes need = part_bytes(slots, D);
    pl.o_bytes = need.o;
    pl.ws_bytes = need.all;
    pl.most_bytes = part_bytes(std::max(slots, most), D).all;
    return true;
}

template <bool BF16, int D, int WAVES, bool PAGED>
hipError_t launch(PromptParams &p, const Plan &pl, hipStream_t stream) {
    using S = Shape<BF16, D, WAVES>;
    void (*kernel)(PromptParams);
    if constexpr (BF16) kernel = &prompt_bf16_kernel<D, WAVES, PAGED>;
    else kernel = &prompt_f32_kernel<D, WAVES, PAGED>;
    const size_t lds = BF16 ? S::kLdsBytes : (WAVES == 1 ? 8 : 4) * S::kTileBytes;
    if (lds > 65536) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)(pl.tiles * p.Hkv * p.splits)), dim3(BF16 ? S::kThreads : 256), lds, stream, p);
    if (p.splits > 1) {
        constexpr int kBlocks = S::kRows / (256 / (D / 4));
        hipLaunchKernelGGL((prompt_join_kernel<BF16, D, S::kRows, PAGED>), dim3((unsigned)(pl.tiles * p.Hkv * kBlocks)), dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}

template <bool PAGED>
hipError_t launch_any(PromptParams &p, const Plan &pl, int32_t D, respec_dtype_t dt, hipStream_t stream) {
    if (dt == RESPEC_F32 && pl.waves == 1) return D == 128 ? launch<false, 128, 1, PAGED>(p, pl, stream) : launch<false, 64, 1, PAGED>(p, pl, stream);
    if (dt == RESPEC_F32) return D == 128 ? launch<false, 128, 4, PAGED>(p, pl, stream) : launch<false, 64, 4, PAGED>(p, pl, stream);
    if (pl.waves == 8) return D == 128 ? launch<true, 128, 8, PAGED>(p, pl, stream) : launch<true, 64, 8, PAGED>(p, pl, stream);
    return D == 128 ? launch<true, 128, 4, PAGED>(p, pl, stream) : launch<true, 64, 4, PAGED>(p, pl, stream);
}

// What the two entry points share.
respec_status_t run(const char *name, PromptParams &p, const void *k, const void *v, int32_t D, float sm_scale, respec_dtype_t dt,
                    void *workspace, size_t workspace_bytes, void *hip_stream, bool paged) {
    if (p.B <= 0 || p.total_q <= 0 || p.max_q <= 0 || p.max_kv <= 0 || p.Hq <= 0 || p.Hkv <= 0)
        return fail(RESPEC_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d total_q=%d max_q=%d max_kv=%d Hq=%d Hkv=%d)", name, p.B,
                    p.total_q, p.max_q, p.max_kv, p.Hq, p.Hkv);
    if (dt != RESPEC_F32 && dt != RESPEC_BF16) return fail(RESPEC_ERR_INVALID_ARG, "%s: unknown dtype %d", name, (int)dt);
    if (p.Hq % p.Hkv != 0) return fail(RESPEC_ERR_INVALID_ARG, "%s: Hq=%d is not a multiple of Hkv=%d", name, p.Hq, p.Hkv);
    if (!std::isfinite(sm_scale)) return fail(RESPEC_ERR_INVALID_ARG, "%s: sm_scale must be finite", name);
    if (D != 64 && D != 128) return fail(RESPEC_ERR_UNSUPPORTED, "%s: head size %d is neither 64 nor 128", name, D);
    if (p.max_kv > INT32_MAX - 256) return fail(RESPEC_ERR_UNSUPPORTED, "%s: max_kv_len must lie 256 below 2^31 - 1 or more", name);
    const int64_t esz = dt == RESPEC_BF16 ? 2 : 4;
    if (p.ld_q < (int64_t)p.Hq * D || p.ld_k < (int64_t)p.Hkv * D || p.ld_v < (int64_t)p.Hkv * D)
        return fail(RESPEC_ERR_INVALID_ARG, "%s: a token stride is smaller than a token", name);
    if (p.ld_k * esz >= (1 << 24) || p.ld_v * esz >= (1 << 24))
        return fail(RESPEC_ERR_UNSUPPORTED, "%s: tokens of K and V must lie less than 2^24 bytes apart", name);
    if (p.ld_q * esz % 16 != 0 || p.ld_k * esz % 16 != 0 || p.ld_v * esz % 16 != 0)
        return fail(RESPEC_ERR_UNSUPPORTED, "%s: token strides must be multiples of 16 bytes", name);
    if (!aligned_to(p.q, 16) || !aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(p.out, 16))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: data pointers must be 16-byte aligned", name);
    Plan pl;
    p.max_q = std::min(p.max_q, p.total_q);
    if (!make_plan(p.B, p.total_q, p.max_q, p.max_kv, p.Hq, p.Hkv, D, dt, pl) || !grid_fits(pl.tiles * p.Hkv * pl.splits, pl.waves == 8 ? 512 : 256))
        return fail(RESPEC_ERR_UNSUPPORTED, "%s: too many rows", name);
    if (!workspace || workspace_bytes < pl.ws_bytes || !aligned_to(workspace, 256))
        return fail(RESPEC_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) needed, got %zu", name, pl.ws_bytes,
                    workspace ? workspace_bytes : (size_t)0);
    p.k = static_cast<const char *>(k);
    p.v = static_cast<const char *>(v);
    p.G = p.Hq / p.Hkv;
    p.splits = pl.splits;
    for (p.g_shift = 0; (1 << p.g_shift) < p.G; ++p.g_shift) {}
    p.g_mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << p.g_shift) - p.G)) / p.G + 1);
    p.g_shift = std::max(1u, p.g_shift);  // (G = 1 divides nothing)
    const uint32_t sign = dt == RESPEC_BF16 ? 0x80008000u : 0x80000000u;
    p.q_and = sm_scale == 0.f ? 0u : ~0u;
    p.q_xor = sm_scale < 0.f ? sign : 0u;
    p.scale2 = sm_scale == 0.f ? 1.f : (float)(std::fabs((double)sm_scale) * 1.4426950408889634074);
    p.part_o = static_cast<float *>(workspace);
    p.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) + pl.o_bytes);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const hipError_t err = paged ? launch_any<true>(p, pl, D, dt, stream) : launch_any<false>(p, pl, D, dt, stream);
    if (err != hipSuccess) return fail(RESPEC_ERR_HIP, "%s: launch failed: %s", name, hipGetErrorString(err));
    clear_error();
    return RESPEC_OK;
}

}  // namespace
}  // namespace respec

extern "C" {

size_t respec_prompt_attention_workspace_bytes(int32_t B, int32_t total_q, int64_t total_kv, int32_t max_q_per_seq, int32_t max_kv_len,
                                               int32_t Hq, int32_t Hkv, int32_t D, respec_dtype_t dt) {
    using namespace respec;
    Plan pl;
    if (total_kv <= 0 || !make_plan(B, total_q, std::min(max_q_per_seq, total_q), max_kv_len, Hq, Hkv, D, dt, pl)) return 0;
    return pl.most_bytes;
}

respec_status_t respec_prompt_attention(const void *q, const void *k, const void *v, const int32_t *q_indptr, const int64_t *kv_indptr,
                                        void *out, float *lse, int32_t B, int32_t total_q, int64_t total_kv, int32_t max_q_per_seq,
                                        int32_t max_kv_len, int32_t Hq, int32_t Hkv, int32_t D, int64_t ld_q, int64_t ld_k, int64_t ld_v,
                                        float sm_scale, respec_dtype_t dt, void *workspace, size_t workspace_bytes, void *hip_stream) {
    using namespace respec;
    if (!q || !k || !v || !q_indptr || !kv_indptr || !out) return fail(RESPEC_ERR_INVALID_ARG, "prompt_attention: null pointer argument");
    if (total_kv <= 0) return fail(RESPEC_ERR_INVALID_ARG, "prompt_attention: total_kv must be positive");
    PromptParams p{};
    p.q = static_cast<const char *>(q);
    p.out = static_cast<char *>(out);
    p.lse = lse;
    p.q_indptr = q_indptr;
    p.kv_indptr = kv_indptr;
    p.ld_q = ld_q;
    p.ld_k = ld_k;
    p.ld_v = ld_v;
    p.total_kv = total_kv;
    p.B = B;
    p.total_q = total_q;
    p.max_q = max_q_per_seq;
    p.max_kv = max_kv_len;
    p.Hq = Hq;
    p.Hkv = Hkv;
    return run("prompt_attention", p, k, v, D, sm_scale, dt, workspace, workspace_bytes, hip_stream, false);
}

respec_status_t respec_prompt_attention_paged(const void *q, const void *k_pages, const void *v_pages, const int32_t *q_indptr,
                                              const int32_t *page_indptr, const int32_t *page_table, const int32_t *kv_len, void *out,
                                              float *lse, int32_t B, int32_t total_q, int32_t num_pages, int32_t page_table_len,
                                              int32_t page_size, int32_t max_q_per_seq, int32_t max_kv_len, int32_t Hq, int32_t Hkv,
                                              int32_t D, int64_t ld_q, float sm_scale, respec_dtype_t dt, void *workspace,
                                              size_t workspace_bytes, void *hip_stream) {
    using namespace respec;
    if (!q || !k_pages || !v_pages || !q_indptr || !page_indptr || !page_table || !kv_len || !out)
        return fail(RESPEC_ERR_INVALID_ARG, "prompt_attention_paged: null pointer argument");
    if (num_pages <= 0 || page_table_len <= 0)
        return fail(RESPEC_ERR_INVALID_ARG, "prompt_attention_paged: sizes must be positive (num_pages=%d page_table_len=%d)", num_pages, page_table_len);
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0)
        return fail(RESPEC_ERR_UNSUPPORTED, "prompt_attention_paged: page size %d is not a power of two in [16, 1024]", page_size);
    PromptParams p{};
    p.q = static_cast<const char *>(q);
    p.out = static_cast<char *>(out);
    p.lse = lse;
    p.q_indptr = q_indptr;
    p.page_indptr = page_indptr;
    p.page_table = page_table;
    p.kv_len = kv_len;
    p.ld_q = ld_q;
    p.ld_k = p.ld_v = (int64_t)Hkv * D;
    p.B = B;
    p.total_q = total_q;
    p.max_q = max_q_per_seq;
    p.max_kv = max_kv_len;
    p.num_pages = num_pages;
    p.table_len = page_table_len;
    p.page_shift = __builtin_ctz((unsigned)page_size);
    p.Hq = Hq;
    p.Hkv = Hkv;
    return run("prompt_attention_paged", p, k_pages, v_pages, D, sm_scale, dt, workspace, workspace_bytes, hip_stream, true);
}

}  // extern "C"
