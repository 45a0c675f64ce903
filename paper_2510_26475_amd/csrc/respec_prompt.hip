// Attention over whole prompts for gfx950: causal, grouped-query heads, packed sequences of different lengths, keys and values in one
// piece or in pages.  This is the forward that fills a cache before the drafts begin and rebuilds it when a sequence moves between
// speculative and plain decoding (Section 5.2); a prompt may come in chunks, its earlier tokens being in the cache already.
//
// The G query heads of a KV head are packed into the rows: packed row r is row r / G, head r % G, so a tile of 128 rows spans
// 128 / G positions, reads K and V once for all its heads and wastes little on the diagonal or on a short prompt.  A wave holds 32
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
constexpr int kWaves16 = 8;           // waves of a work-group in bf16
constexpr int kSplitTiles = 512;      // work-groups below which a call is split

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
    int32_t splits, tiles;   // parts of a tile's keys; bound of the row tiles of a KV head
    uint32_t q_and, q_xor;   // on the bits of q: a negative scale is taken out of it, a zero one makes it zero
    float scale2;            // |sm_scale| * log2(e)
    float *part_o;           // [tiles * Hkv * splits][rows][D]
    float *part_ml;          // [tiles * Hkv * splits][rows][2]
};

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

template <bool BF16, int D, int WAVES, bool PAGED>
__device__ inline bool find_job(const PromptParams &p, Job &j) {
    using S = Shape<BF16, D, WAVES>;
    j.head = blockIdx.x % p.Hkv;
    const int rest = blockIdx.x / p.Hkv, split = rest % p.splits;
    j.number = blockIdx.x;
    if (!find_tile(p.q_indptr, p.B, p.total_q, p.max_q, p.G, S::kRows, rest / p.splits, j.tile)) return false;
    j.tile.index = j.tile.tiles - 1 - j.tile.index;  // (the longest first)
    if constexpr (PAGED) {
        j.kv0 = max(0, min(p.page_indptr[j.tile.b], p.table_len));
        const int64_t pages = max((int64_t)0, (int64_t)min(p.page_indptr[j.tile.b + 1], p.table_len) - j.kv0);
        j.L = (int)max((int64_t)0, min(min((int64_t)p.kv_len[j.tile.b], pages << p.page_shift), (int64_t)p.max_kv));
    } else {
        j.kv0 = max((int64_t)0, min(p.kv_indptr[j.tile.b], p.total_kv));
        j.L = (int)max((int64_t)0, min(min(p.kv_indptr[j.tile.b + 1], p.total_kv) - j.kv0, (int64_t)p.max_kv));
    }
    j.L = __builtin_amdgcn_readfirstlane(j.L);
    j.n_rows = j.tile.R * p.G;
    j.row0 = j.tile.index * S::kRows;
    const int last = min(j.row0 + S::kRows, j.n_rows) - 1;
    const int end = j.L - j.tile.R + last / p.G + 1;  // the work-group's last row sees most
    const int tiles = max(0, (end + S::kKeys - 1) / S::kKeys);
    j.t_begin = (int)((int64_t)tiles * split / p.splits);
    j.t_end = (int)((int64_t)tiles * (split + 1) / p.splits);
    j.all = j.L - j.tile.R + j.row0 / p.G + 1;
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
    const int i = clamped / p.G;
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
    for (int x = 0; x < CHUNKS / 2; ++x) {
        qf[x] = *reinterpret_cast<const u32x4 *>(qp + x * 32);
        for (int w = 0; w < 4; ++w) qf[x][w] = (qf[x][w] & p.q_and) ^ p.q_xor;
    }
}

typedef const __attribute__((address_space(4))) int32_t *ConstInts;  // (read through the scalar cache; nothing writes it meanwhile)

// Moves K or V pieces from global memory into registers: key wave * kWaveKeys + lane / kChunks + i * (keys of all waves), piece
// lane % kChunks.  The keys of a load lie in one page, so what differs between lanes is a 32-bit offset.  Keys past the end are the
// last one's (they are never seen).
template <bool BF16, int D, int WAVES, bool PAGED>
struct Mover {
    using S = Shape<BF16, D, WAVES>;
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
    __device__ int64_t row(int n) const {  // of a key in K and V (uniform)
        if constexpr (PAGED) {
            const int64_t page = max(0, min(table[n >> shift], num_pages - 1));
            return (page << shift) + (n & ((1 << shift) - 1));
        } else {
            return kv0 + n;
        }
    }
    template <bool V>
    __device__ void load(int t, u32x4 (&x)[S::kLoads]) const {
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i) {
            const int n = max(0, min(t * S::kKeys + i * (WAVES * S::kWaveKeys) + wave * S::kWaveKeys, L - 1));  // (uniform)
            const uint32_t ld = (uint32_t)(V ? ld_v : ld_k);
            const uint32_t off = __umul24((uint32_t)min(my_key, L - 1 - n), ld) + my_piece;
            const char *base = (V ? v : k) + row(n) * (V ? ld_v : ld_k);
            x[i] = *reinterpret_cast<const u32x4 *>(base + off);
        }
    }
    // The same for a tile that lies in the sequence as a whole.
    template <bool V>
    __device__ void load_whole(int t, u32x4 (&x)[S::kLoads]) const {
        const int64_t ld = V ? ld_v : ld_k;
        const char *const from = V ? v : k;
        if constexpr (PAGED) {
            const uint32_t off = __umul24((uint32_t)my_key, (uint32_t)ld) + my_piece;
#pragma unroll
            for (int i = 0; i < S::kLoads; ++i)
                x[i] = *reinterpret_cast<const u32x4 *>(from + row(t * S::kKeys + i * (WAVES * S::kWaveKeys) + wave * S::kWaveKeys) * ld + off);
        } else {
            const char *const base = from + (kv0 + (int64_t)t * S::kKeys) * ld;
            uint32_t off = __umul24((uint32_t)(wave * S::kWaveKeys + my_key), (uint32_t)ld) + my_piece;
#pragma unroll
            for (int i = 0; i < S::kLoads; ++i) {
                x[i] = *reinterpret_cast<const u32x4 *>(base + off);
                off += (uint32_t)ld * (WAVES * S::kWaveKeys);
            }
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
                              int not_finite) {
    using S = Shape<BF16, D, WAVES>;
    const int64_t slot = (int64_t)j.number * S::kRows + wave * 32 + col;
    if (r.exists && p.splits > 1) {
        if (half == 0) *reinterpret_cast<floatx2 *>(p.part_ml + slot * 2) = floatx2{m, l};
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; x += 4)
                *reinterpret_cast<floatx4 *>(p.part_o + slot * D + d * 32 + 2 * x + 4 * half) = floatx4{o[d][x], o[d][x + 1], o[d][x + 2], o[d][x + 3]};
    } else if (r.exists) {
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;  // (no visible key: zero; NaN stays)
        char *op = p.out + (r.token * p.Hq + r.head) * (int64_t)S::kRowBytes;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; x += 4) {  // four d in a row
                const floatx4 y = {o[d][x] * inv, o[d][x + 1] * inv, o[d][x + 2] * inv, o[d][x + 3] * inv};
                const int at = d * 32 + 2 * x + 4 * half;
                if constexpr (BF16) {
                    const bf16x2 a = __builtin_convertvector(floatx2{y[0], y[1]}, bf16x2), c = __builtin_convertvector(floatx2{y[2], y[3]}, bf16x2);
                    *reinterpret_cast<u32x2 *>(op + at * 2) = u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c)};
                } else {
                    *reinterpret_cast<floatx4 *>(op + at * 4) = y;
                }
            }
        if (p.lse && half == 0) p.lse[r.token * p.Hq + r.head] = l == 0.f ? -INFINITY : m * 0.693147180559945309f + logf(l);
    }
    if (not_finite == 0) return;  // (uniform)
    // The values that put_v left out, added to what the work-group has written: a row and a d of it per thread.
    __syncthreads();
    const int first_key = max(j.t_begin, j.all / S::kKeys) * S::kKeys, end_key = j.t_end * S::kKeys;
    for (int e = threadIdx.x; e < S::kRows * D; e += S::kThreads) {
        const int row = j.row0 + e / D, d = e % D;
        if (row >= j.n_rows) break;
        const int sees = min(end_key, j.L - j.tile.R + row / p.G + 1);
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
            char *op = p.out + (((j.tile.q0 + row / p.G) * p.Hq + j.head * p.G + row % p.G) * (int64_t)D + d) * S::kSize;
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

// fp32: one tile of 32 keys after the other.
template <int D, bool PAGED>
__global__ __launch_bounds__(256, 2) void prompt_f32_kernel(PromptParams p) {
    constexpr int kWaves = 4;
    using S = Shape<false, D, kWaves>;
    extern __shared__ __align__(16) char lds[];  // two tiles of K, two of V
    __shared__ int sh_not_finite;
    char *const lds_k = lds, *const lds_v = lds + 2 * S::kTileBytes;
    Job job;
    if (!find_job<false, D, kWaves, PAGED>(p, job)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    const RowOf row = row_of(p, job, wave, col);
    u32x4 qf[S::kChunks / 2];
    load_q<S::kChunks>(p, row, D, S::kSize, half, qf);
    const Mover<false, D, kWaves, PAGED> mover(p, job, wave, lane);
    if (threadIdx.x == 0) sh_not_finite = 0;
    __syncthreads();

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
    if (job.t_begin < job.t_end) {  // (uniform)
        mover.template load<false>(job.t_begin, kr);
        mover.template load<true>(job.t_begin, vr);
        put(0, job.t_begin);
        __syncthreads();
    }
    for (int t = job.t_begin; t < job.t_end; ++t) {
        const int buffer = (t - job.t_begin) & 1;
        if (t + 1 < job.t_end) {
            mover.template load<false>(t + 1, kr);
            mover.template load<true>(t + 1, vr);
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
        if (t + 1 < job.t_end) put(buffer ^ 1, t + 1);
        __syncthreads();
    }
    finish<false, D, kWaves, PAGED>(p, job, row, wave, half, col, o, m, sum_of_halves(l), sh_not_finite);
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

// bf16: the scores of tile t+1 are multiplied while the exponentials of tile t are computed.  K is one tile ahead of V in LDS, and the
// loop is written for two tiles, so that a tile's buffer is a constant and every LDS address one of twelve that a lane keeps.
template <int D, int WAVES, bool PAGED>
__global__ __launch_bounds__(WAVES * 64, 2) void prompt_bf16_kernel(PromptParams p) {
    using S = Shape<true, D, WAVES>;
    extern __shared__ __align__(16) char lds[];  // two tiles of K, two of V
    __shared__ int sh_not_finite;
    Job job;
    if (!find_job<true, D, WAVES, PAGED>(p, job)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    const RowOf row = row_of(p, job, wave, col);
    u32x4 qf[S::kChunks / 2];
    load_q<S::kChunks>(p, row, D, S::kSize, half, qf);
    const Mover<true, D, WAVES, PAGED> mover(p, job, wave, lane);
    if (threadIdx.x == 0) sh_not_finite = 0;
    __syncthreads();

    // Where this lane reads: a key's pieces of K; for V the transposing read's sixteen lanes address four keys by sixteen d.
    int k_at[S::kChunks / 2], v_at[S::kDTiles];
#pragma unroll
    for (int x = 0; x < S::kChunks / 2; ++x) k_at[x] = col * S::kRowBytes + k_piece<true, D>(col, 2 * x + half) * 16;
    const int i16 = lane & 15, v_key = half * 4 + (i16 >> 2), d0 = ((lane & 16) + 4 * (i16 & 3)) * 2;
#pragma unroll
    for (int d = 0; d < S::kDTiles; ++d) v_at[d] = v_key * S::kRowBytes + v_piece<true, D>(v_key, (d * 64 + d0) >> 4) * 16 + (d0 & 15);

    floatx16 o[S::kDTiles];
#pragma unroll
    for (int d = 0; d < S::kDTiles; ++d)
        for (int x = 0; x < 16; ++x) o[d][x] = 0.f;
    float m = -INFINITY, ref = 0.f, l = 0.f;
    u32x4 kr[S::kLoads], vr[S::kLoads];
    floatx16 s_even[S::kBlocks], s_odd[S::kBlocks];

    auto scores = [&](auto buffer, floatx16(&s)[S::kBlocks]) __attribute__((always_inline)) {
        constexpr int kAt = decltype(buffer)::value * S::kTileBytes;
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
            for (int x = 0; x < S::kChunks / 2; ++x) {
                const bf16x8 a = *reinterpret_cast<const bf16x8 *>(lds + k_at[x] + (kAt + b * 32 * S::kRowBytes));
                const floatx16 none{};
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, qf[x]), x == 0 ? none : s[b], 0, 0, 0);
            }
    };
    // Probabilities of sixteen keys as the B operand of the second product: slot j is key 8 (j / 4) + 4 half + j % 4 of them.
    auto weights = [&](const floatx16 &s, int h) __attribute__((always_inline)) {
        bf16x8 pf;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float a = __builtin_amdgcn_exp2f(fmaf(s[h * 8 + j], p.scale2, -ref)), c = __builtin_amdgcn_exp2f(fmaf(s[h * 8 + j + 1], p.scale2, -ref));
            l += a;
            l += c;
            const bf16x2 two = __builtin_convertvector(floatx2{a, c}, bf16x2);
            pf[j] = two[0];
            pf[j + 1] = two[1];
        }
        return pf;
    };
    auto product = [&](auto buffer, int b, int h, const bf16x8 &pf) __attribute__((always_inline)) {
        constexpr int kAt = (2 + decltype(buffer)::value) * S::kTileBytes;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d) {
            s16x4 vt[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                vt[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTr)(lds + v_at[d] + (kAt + (b * 32 + h * 16 + j * 8) * S::kRowBytes)));
            const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vt[0], vt[1], 0, 1, 2, 3, 4, 5, 6, 7));
            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pf, o[d], 0, 0, 0);
        }
    };
    auto largest = [&](const floatx16(&s)[S::kBlocks]) __attribute__((always_inline)) {
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
            for (int x = b == 0; x < 16; ++x) top = fmaxf(top, s[b][x]);
        return max_of_halves(top) * p.scale2;
    };
    auto mask = [&](int t, floatx16(&s)[S::kBlocks]) __attribute__((always_inline)) {
        if ((t + 1) * S::kKeys > row.wave_all)
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) mask_scores(s[b], t * S::kKeys + b * 32, half, row.lim);
    };
    auto rescale = [&](float top) __attribute__((always_inline)) {
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
    // Tile t, its scores in s (the maximum taken into account), V in `buffer`, the next tile's K in the other one; all rows see both
    // tiles.  One block of code: the matrix unit has the scores of the next tile and the second product of this one to do while
    // the exponentials of this one and the maximum of the next are computed.
    auto both = [&](auto buffer, int t, floatx16(&s)[S::kBlocks], floatx16(&next)[S::kBlocks]) __attribute__((always_inline)) {
        constexpr int kB = decltype(buffer)::value;
        mover.template load_whole<false>(t + 2, kr);
        mover.template load_whole<true>(t + 1, vr);
        // Written in the order it is to run in: a product, an LDS read kAhead products before its use, and a share of the rest.
        constexpr int kAhead = 4, kFirst = S::kBlocks * S::kChunks / 2, kSecond = 2 * S::kBlocks * S::kDTiles;
        constexpr int kPairs = 16 * S::kBlocks / 2;  // of probabilities; those of the last sixteen keys are not needed before the last products
        bf16x8 ahead[kAhead];
        u32x4 pf[2 * S::kBlocks];
        auto read = [&](auto i_) __attribute__((always_inline)) {
            constexpr int i = decltype(i_)::value;
            if constexpr (i < kFirst) {
                constexpr int b = i % S::kBlocks, x = i / S::kBlocks;
                ahead[i % kAhead] = *reinterpret_cast<const bf16x8 *>(lds + k_at[x] + ((1 - kB) * S::kTileBytes + b * 32 * S::kRowBytes));
            } else if constexpr (i < kFirst + kSecond) {
                constexpr int g = (i - kFirst) / S::kDTiles, d = (i - kFirst) % S::kDTiles;
                s16x4 vt[2];
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    vt[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsTr)(lds + v_at[d] + ((2 + kB) * S::kTileBytes + (g * 16 + j * 8) * S::kRowBytes)));
                ahead[i % kAhead] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vt[0], vt[1], 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        auto pair = [&](auto n_) __attribute__((always_inline)) {
            constexpr int n = decltype(n_)::value, g = n / 4, j = n % 4 * 2;
            const floatx16 &from = s[g / 2];
            const float a = __builtin_amdgcn_exp2f(fmaf(from[g % 2 * 8 + j], p.scale2, -ref));
            const float c = __builtin_amdgcn_exp2f(fmaf(from[g % 2 * 8 + j + 1], p.scale2, -ref));
            l += a;
            l += c;
            pf[g][j / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, c}, bf16x2));
        };
        float top = -INFINITY;
        each<kAhead>([&](auto i) __attribute__((always_inline)) { read(i); });
        __builtin_amdgcn_sched_barrier(0);
        each<kFirst + kSecond>([&](auto i_) __attribute__((always_inline)) {
            constexpr int i = decltype(i_)::value;
            if constexpr (i < kFirst) {
                constexpr int b = i % S::kBlocks, x = i / S::kBlocks;
                const floatx16 none{};
                next[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[i % kAhead], __builtin_bit_cast(bf16x8, qf[x]), x == 0 ? none : next[b], 0, 0, 0);
            } else {
                constexpr int g = (i - kFirst) / S::kDTiles, d = (i - kFirst) % S::kDTiles;
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[i % kAhead], __builtin_bit_cast(bf16x8, pf[g]), o[d], 0, 0, 0);
            }
            read(std::integral_constant<int, i + kAhead>{});
            // pairs: two in three products of the first kind, the rest in the second kind's first ones; then the maximum
            constexpr int kShare = kPairs * 5 / 8;
            if constexpr (i < kFirst) {
                constexpr int from = i * kShare / kFirst, to = (i + 1) * kShare / kFirst;
                each<to - from>([&](auto n) __attribute__((always_inline)) { pair(std::integral_constant<int, from + decltype(n)::value>{}); });
            } else {
                constexpr int n = kShare + i - kFirst, rest = kPairs - kShare, k = i - kFirst - rest, kLast = kSecond - rest;
                if constexpr (n < kPairs) pair(std::integral_constant<int, n>{});
                else {
                    constexpr int from = 16 * S::kBlocks * k / kLast, to = 16 * S::kBlocks * (k + 1) / kLast;
#pragma unroll
                    for (int x = from; x < to; ++x) top = fmaxf(top, next[x / 16][x % 16]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        top = max_of_halves(top) * p.scale2;
        rescale(top);
        mover.put_k(lds + kB * S::kTileBytes, kr);
        mover.put_v(lds + (3 - kB) * S::kTileBytes, vr, false, &sh_not_finite);
        __syncthreads();
    };
    // Any tile, its scores in s: the second product, then the next tile's scores.
    auto one = [&](auto buffer, int t, floatx16(&s)[S::kBlocks], floatx16(&next)[S::kBlocks]) __attribute__((always_inline)) {
        constexpr int kB = decltype(buffer)::value;
        const std::integral_constant<int, kB> here{};
        const std::integral_constant<int, 1 - kB> there{};
        const bool more = t + 1 < job.t_end;
        if (t + 2 < job.t_end) mover.template load<false>(t + 2, kr);
        if (more) mover.template load<true>(t + 1, vr);
        if (t * S::kKeys < row.wave_sees)
#pragma unroll
            for (int i = 0; i < 2 * S::kBlocks; ++i) product(here, i / 2, i % 2, weights(s[i / 2], i % 2));
        if (more && (t + 1) * S::kKeys < row.wave_sees) {
            scores(there, next);
            mask(t + 1, next);
            rescale(largest(next));
        }
        if (t + 2 < job.t_end) mover.put_k(lds + kB * S::kTileBytes, kr);
        if (more) mover.put_v(lds + (3 - kB) * S::kTileBytes, vr, (t + 2) * S::kKeys > job.all, &sh_not_finite);
        __syncthreads();
    };

    int t = job.t_begin;
    if (t < job.t_end) {  // (uniform)
        mover.template load<false>(t, kr);
        mover.template load<true>(t, vr);
        mover.put_k(lds, kr);
        mover.put_v(lds + 2 * S::kTileBytes, vr, (t + 1) * S::kKeys > job.all, &sh_not_finite);
        mover.template load<false>(min(t + 1, job.t_end - 1), kr);
        mover.put_k(lds + S::kTileBytes, kr);
        __syncthreads();
        if (t * S::kKeys < row.wave_sees) {
            scores(std::integral_constant<int, 0>{}, s_even);
            mask(t, s_even);
            rescale(largest(s_even));
        }
        __syncthreads();  // (the first tile's K is read by all before it is written over)
    }
    const int seen_by_all = min(job.t_end, max(job.all, 0) / S::kKeys);  // tiles
    for (; t + 3 < seen_by_all; t += 2) {  // (the loads are two tiles ahead)
        both(std::integral_constant<int, 0>{}, t, s_even, s_odd);
        both(std::integral_constant<int, 1>{}, t + 1, s_odd, s_even);
    }
    for (; t < job.t_end; t += 2) {
        one(std::integral_constant<int, 0>{}, t, s_even, s_odd);
        if (t + 1 < job.t_end) one(std::integral_constant<int, 1>{}, t + 1, s_odd, s_even);
    }
    finish<true, D, WAVES, PAGED>(p, job, row, wave, half, col, o, m, sum_of_halves(l), sh_not_finite);
}

// Joins the parts of a tile's keys: a thread per packed row and four elements.
template <bool BF16, int D, int ROWS>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptParams p) {
    constexpr int kQuads = D / 4, kPerBlock = 256 / kQuads;  // rows of a work-group
    constexpr int kBlocks = ROWS / kPerBlock;                // work-groups of a tile
    const int piece = blockIdx.x % kBlocks, head = blockIdx.x / kBlocks % p.Hkv, number = blockIdx.x / kBlocks / p.Hkv;
    Tile tile;
    if (!find_tile(p.q_indptr, p.B, p.total_q, p.max_q, p.G, ROWS, number, tile)) return;
    tile.index = tile.tiles - 1 - tile.index;
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
    const int i_row = packed / p.G, q_head = head * p.G + packed % p.G;
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
};

// The split: as many parts of the keys as fill the device twice, no part below 512 keys.
bool make_plan(int32_t B, int32_t total_q, int32_t max_q, int32_t max_kv, int32_t Hq, int32_t Hkv, int32_t D, respec_dtype_t dt, Plan &pl) {
    if (B <= 0 || total_q <= 0 || max_q <= 0 || max_kv <= 0 || Hq <= 0 || Hkv <= 0) return false;
    if (Hq % Hkv != 0 || (D != 64 && D != 128) || (dt != RESPEC_F32 && dt != RESPEC_BF16)) return false;
    const int32_t G = Hq / Hkv;
    if ((int64_t)std::min(max_q, total_q) * G >= (1 << 30)) return false;
    pl.waves = dt == RESPEC_BF16 ? kWaves16 : 4;
    const int rows = pl.waves * 32;
    pl.tiles = tiles_bound(B, total_q, std::min(max_q, total_q), G, rows);
    const int64_t groups = pl.tiles * Hkv;
    pl.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>({kMaxSplits, kSplitTiles / groups, max_kv / 512}));
    const size_t slots = pl.splits > 1 ? (size_t)groups * pl.splits * rows : 0;
    pl.o_bytes = round_up(slots * D * sizeof(float), 256);
    pl.ws_bytes = std::max<size_t>(256, pl.o_bytes + round_up(slots * 2 * sizeof(float), 256));
    return true;
}

template <bool BF16, int D, bool PAGED>
hipError_t launch(PromptParams &p, const Plan &pl, hipStream_t stream) {
    using S = Shape<BF16, D, BF16 ? kWaves16 : 4>;
    const size_t lds = 4 * S::kTileBytes;
    void (*kernel)(PromptParams);
    if constexpr (BF16) kernel = &prompt_bf16_kernel<D, kWaves16, PAGED>;
    else kernel = &prompt_f32_kernel<D, PAGED>;
    if (lds > 65536) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)(pl.tiles * p.Hkv * p.splits)), dim3(S::kThreads), lds, stream, p);
    if (p.splits > 1) {
        constexpr int kBlocks = S::kRows / (256 / (D / 4));
        hipLaunchKernelGGL((prompt_join_kernel<BF16, D, S::kRows>), dim3((unsigned)(pl.tiles * p.Hkv * kBlocks)), dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}

template <bool PAGED>
hipError_t launch_any(PromptParams &p, const Plan &pl, int32_t D, respec_dtype_t dt, hipStream_t stream) {
    if (dt == RESPEC_BF16) return D == 128 ? launch<true, 128, PAGED>(p, pl, stream) : launch<true, 64, PAGED>(p, pl, stream);
    return D == 128 ? launch<false, 128, PAGED>(p, pl, stream) : launch<false, 64, PAGED>(p, pl, stream);
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
    if (!make_plan(p.B, p.total_q, p.max_q, p.max_kv, p.Hq, p.Hkv, D, dt, pl) || pl.tiles * p.Hkv * pl.splits > (1 << 26))
        return fail(RESPEC_ERR_UNSUPPORTED, "%s: too many rows", name);
    if (!workspace || workspace_bytes < pl.ws_bytes || !aligned_to(workspace, 256))
        return fail(RESPEC_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) needed, got %zu", name, pl.ws_bytes,
                    workspace ? workspace_bytes : (size_t)0);
    p.k = static_cast<const char *>(k);
    p.v = static_cast<const char *>(v);
    p.G = p.Hq / p.Hkv;
    p.splits = pl.splits;
    p.tiles = (int32_t)pl.tiles;
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
    return pl.ws_bytes;
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
