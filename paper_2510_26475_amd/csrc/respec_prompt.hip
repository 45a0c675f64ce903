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
    static constexpr int kDTiles = D / 32;
    static_assert(kKeys * kChunks % kThreads == 0, "whole pieces per thread");
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

__device__ inline float other_half(float x) {  // the value of lane ^ 32
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float((threadIdx.x & 32) ? a[0] : a[1]);
}

template <bool BF16, int D, int WAVES, bool PAGED>
__global__ __launch_bounds__(WAVES * 64, 2) void prompt_kernel(PromptParams p) {
    using S = Shape<BF16, D, WAVES>;
    extern __shared__ __align__(16) char lds[];  // two tiles of K, two of V
    char *const lds_k = lds, *const lds_v = lds + 2 * S::kTileBytes;
    __shared__ int sh_not_finite;

    const int head = blockIdx.x % p.Hkv, rest = blockIdx.x / p.Hkv;
    const int split = rest % p.splits;
    Tile tile;
    if (!find_tile(p.q_indptr, p.B, p.total_q, p.max_q, p.G, S::kRows, rest / p.splits, tile)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5, col = lane & 31;
    tile.index = tile.tiles - 1 - tile.index;  // (the longest first)

    // the sequence's keys
    int64_t kv0;
    int L;
    if constexpr (PAGED) {
        kv0 = max(0, min(p.page_indptr[tile.b], p.table_len));
        const int64_t pages = max((int64_t)0, (int64_t)min(p.page_indptr[tile.b + 1], p.table_len) - kv0);
        L = (int)max((int64_t)0, min(min((int64_t)p.kv_len[tile.b], pages << p.page_shift), (int64_t)p.max_kv));
    } else {
        kv0 = max((int64_t)0, min(p.kv_indptr[tile.b], p.total_kv));
        L = (int)max((int64_t)0, min(min(p.kv_indptr[tile.b + 1], p.total_kv) - kv0, (int64_t)p.max_kv));
    }
    // this lane's row: it sees keys 0 .. lim-1
    const int n_rows = tile.R * p.G;
    const int row0 = tile.index * S::kRows;
    const int packed = row0 + wave * 32 + col;
    const bool exists = packed < n_rows;
    const int i_row = min(packed, n_rows - 1) / p.G, g = min(packed, n_rows - 1) - i_row * p.G;
    const int lim = L - tile.R + i_row + 1;
    const int64_t token = tile.q0 + i_row;
    const int q_head = head * p.G + g;
    const int last = min(row0 + S::kRows, n_rows) - 1;
    const int end = L - tile.R + last / p.G + 1;  // the work-group's last row sees most
    const int all_tiles = max(0, (end + S::kKeys - 1) / S::kKeys);
    const int t_begin = (int)((int64_t)all_tiles * split / p.splits), t_end = (int)((int64_t)all_tiles * (split + 1) / p.splits);
    const int wave_last = min(row0 + wave * 32 + 31, n_rows - 1), wave_first = min(row0 + wave * 32, n_rows - 1);
    const int wave_sees = __builtin_amdgcn_readfirstlane(L - tile.R + wave_last / p.G + 1);    // keys that some row of the wave sees
    const int wave_all = __builtin_amdgcn_readfirstlane(L - tile.R + wave_first / p.G + 1);    // that all of them see

    const int block_all = L - tile.R + row0 / p.G + 1;  // keys that all rows of the work-group see
    if (threadIdx.x == 0) sh_not_finite = 0;
    __syncthreads();

    // Q^T as the B operand: this lane's column is its row, its contraction slots the pieces 2x + half of the row
    u32x4 qf[S::kChunks / 2];
    {
        const char *qp = p.q + (token * p.ld_q + (int64_t)q_head * D) * S::kSize + half * 16;
#pragma unroll
        for (int x = 0; x < S::kChunks / 2; ++x) {
            qf[x] = *reinterpret_cast<const u32x4 *>(qp + x * 32);
            for (int w = 0; w < 4; ++w) qf[x][w] = (qf[x][w] & p.q_and) ^ p.q_xor;
        }
    }

    // the pieces that this thread moves: key thread / kChunks + i * kThreads / kChunks, piece thread % kChunks
    constexpr int kKeyStep = S::kThreads / S::kChunks;
    const int my_key = threadIdx.x / S::kChunks, my_piece = threadIdx.x % S::kChunks;
    u32x4 kr[S::kLoads], vr[S::kLoads];
    int32_t page[PAGED ? S::kLoads : 1];
    const int64_t head_bytes = (int64_t)head * S::kRowBytes + my_piece * 16;
    auto look_up = [&](int t) __attribute__((always_inline)) {
        if constexpr (PAGED) {
#pragma unroll
            for (int i = 0; i < S::kLoads; ++i) {
                const int n = max(0, min(t * S::kKeys + my_key + i * kKeyStep, L - 1));
                page[i] = p.page_table[kv0 + (n >> p.page_shift)];
            }
        }
    };
    auto request = [&](int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i) {
            const int n = max(0, min(t * S::kKeys + my_key + i * kKeyStep, L - 1));  // (keys past the end: the last one's, never seen)
            int64_t at;
            if constexpr (PAGED) at = ((int64_t)max(0, min(page[i], p.num_pages - 1)) << p.page_shift) + (n & ((1 << p.page_shift) - 1));
            else at = kv0 + n;
            kr[i] = *reinterpret_cast<const u32x4 *>(p.k + at * p.ld_k * S::kSize + head_bytes);
            vr[i] = *reinterpret_cast<const u32x4 *>(p.v + at * p.ld_v * S::kSize + head_bytes);
        }
    };
    auto put = [&](int buffer, int t) __attribute__((always_inline)) {
        if ((t + 1) * S::kKeys > block_all) {
            // Some row does not see all of the tile.  A product would carry a value that is not finite to it all the same: such
            // values count as zero here and reach the rows that see them at the end.
            bool bad = false;
#pragma unroll
            for (int i = 0; i < S::kLoads; ++i)
                for (int w = 0; w < 4; ++w) {
                    const bool hi = (vr[i][w] & 0x7f800000u) == 0x7f800000u, lo = BF16 && (vr[i][w] & 0x7f80u) == 0x7f80u;
                    bad |= hi || lo;
                    vr[i][w] &= (hi ? (BF16 ? 0xffffu : 0u) : ~0u) & (lo ? 0xffff0000u : ~0u);
                }
            if (bad) sh_not_finite = 1;
        }
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i) {
            const int key = my_key + i * kKeyStep;
            *reinterpret_cast<u32x4 *>(lds_k + buffer * S::kTileBytes + key * S::kRowBytes + k_piece<BF16, D>(key, my_piece) * 16) = kr[i];
            *reinterpret_cast<u32x4 *>(lds_v + buffer * S::kTileBytes + key * S::kRowBytes + v_piece<BF16, D>(key, my_piece) * 16) = vr[i];
        }
    };

    floatx16 o[S::kDTiles];
#pragma unroll
    for (int d = 0; d < S::kDTiles; ++d)
        for (int x = 0; x < 16; ++x) o[d][x] = 0.f;
    float m = -INFINITY, l = 0.f;

    if (t_begin < t_end) {  // (uniform)
        look_up(t_begin);
        request(t_begin);
        if (t_begin + 1 < t_end) look_up(t_begin + 1);
        put(0, t_begin);
        __syncthreads();
    }
    for (int t = t_begin; t < t_end; ++t) {
        const int buffer = (t - t_begin) & 1;
        if (t + 1 < t_end) {
            request(t + 1);
            if (t + 2 < t_end) look_up(t + 2);
        }
        if (t * S::kKeys < wave_sees) {
            const char *kb = lds_k + buffer * S::kTileBytes, *vb = lds_v + buffer * S::kTileBytes;
            floatx16 s[S::kBlocks];
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b) {
                for (int x = 0; x < 16; ++x) s[b][x] = 0.f;
                const int key = b * 32 + col;
#pragma unroll
                for (int x = 0; x < S::kChunks / 2; ++x) {
                    const u32x4 a = *reinterpret_cast<const u32x4 *>(kb + key * S::kRowBytes + k_piece<BF16, D>(key, 2 * x + half) * 16);
                    if constexpr (BF16) {
                        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, qf[x]), s[b], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            s[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[y]), __uint_as_float(qf[x][y]), s[b], 0, 0, 0);
                    }
                }
            }
            if ((t + 1) * S::kKeys > wave_all) {  // score x of block b is key 32 b + 8 (x / 4) + 4 half + x % 4
#pragma unroll
                for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                    for (int x = 0; x < 16; ++x)
                        if (t * S::kKeys + b * 32 + 8 * (x / 4) + 4 * half + x % 4 >= lim) s[b][x] = -INFINITY;
            }
            float top = s[0][0];
#pragma unroll
            for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                for (int x = 0; x < 16; ++x) top = fmaxf(top, s[b][x]);
            top = fmaxf(top, other_half(top)) * p.scale2;
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
            for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    s[b][x] = __builtin_amdgcn_exp2f(fmaf(s[b][x], p.scale2, -ref));
                    l += s[b][x];
                }
            if constexpr (BF16) {
                // sixteen keys at a time: slot j of this lane is key 8 (j / 4) + 4 half + j % 4 of them.  V^T comes by the transposing
                // read: the sixteen lanes of a group address four keys by sixteen d and receive one d of the four keys each.
                const int i16 = lane & 15, d0 = (lane & 16) + 4 * (i16 & 3);
#pragma unroll
                for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        bf16x8 pf;
#pragma unroll
                        for (int j = 0; j < 8; j += 2) {
                            const bf16x2 two = __builtin_convertvector(floatx2{s[b][h * 8 + j], s[b][h * 8 + j + 1]}, bf16x2);
                            pf[j] = two[0];
                            pf[j + 1] = two[1];
                        }
#pragma unroll
                        for (int d = 0; d < S::kDTiles; ++d) {
                            s16x4 vt[2];
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const int key = b * 32 + h * 16 + j * 8 + half * 4 + (i16 >> 2), at = (d * 32 + d0) * 2;
                                vt[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                    (LdsTr)(vb + key * S::kRowBytes + v_piece<BF16, D>(key, at >> 4) * 16 + (at & 15)));
                            }
                            const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vt[0], vt[1], 0, 1, 2, 3, 4, 5, 6, 7));
                            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pf, o[d], 0, 0, 0);
                        }
                    }
            } else {
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    const int key = 8 * (x / 4) + 4 * half + x % 4;
#pragma unroll
                    for (int d = 0; d < S::kDTiles; ++d)
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float *>(vb + key * S::kRowBytes + (d * 32 + col) * 4),
                                                                    s[0][x], o[d], 0, 0, 0);
                }
            }
        }
        if (t + 1 < t_end) put(buffer ^ 1, t + 1);
        __syncthreads();
    }
    l += other_half(l);

    const int64_t slot = (int64_t)blockIdx.x * S::kRows + wave * 32 + col;
    if (exists && p.splits > 1) {
        if (half == 0) *reinterpret_cast<floatx2 *>(p.part_ml + slot * 2) = floatx2{m, l};
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; x += 4)
                *reinterpret_cast<floatx4 *>(p.part_o + slot * D + d * 32 + 2 * x + 4 * half) = floatx4{o[d][x], o[d][x + 1], o[d][x + 2], o[d][x + 3]};
    } else if (exists) {
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;  // (no visible key: zero; NaN stays)
        char *op = p.out + (token * p.Hq + q_head) * (int64_t)S::kRowBytes;
#pragma unroll
        for (int d = 0; d < S::kDTiles; ++d)
#pragma unroll
            for (int x = 0; x < 16; x += 4) {  // four d in a row
                const floatx4 r = {o[d][x] * inv, o[d][x + 1] * inv, o[d][x + 2] * inv, o[d][x + 3] * inv};
                const int at = d * 32 + 2 * x + 4 * half;
                if constexpr (BF16) {
                    const bf16x2 a = __builtin_convertvector(floatx2{r[0], r[1]}, bf16x2), c = __builtin_convertvector(floatx2{r[2], r[3]}, bf16x2);
                    *reinterpret_cast<u32x2 *>(op + at * 2) = u32x2{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c)};
                } else {
                    *reinterpret_cast<floatx4 *>(op + at * 4) = r;
                }
            }
        if (p.lse && half == 0) p.lse[token * p.Hq + q_head] = l == 0.f ? -INFINITY : m * 0.693147180559945309f + logf(l);
    }

    if (sh_not_finite == 0) return;  // (uniform: written before the last barrier)
    // The values left out above, added to what the work-group has written: a row and a d of it per thread.
    __syncthreads();
    const int first_key = max(t_begin, block_all / S::kKeys) * S::kKeys, end_key = t_end * S::kKeys;
    for (int e = threadIdx.x; e < S::kRows * D; e += S::kThreads) {
        const int r = row0 + e / D, d = e % D;
        if (r >= n_rows) break;
        const int sees = min(end_key, L - tile.R + r / p.G + 1);
        float sum = 0.f;
        for (int n = first_key; n < sees; ++n) {
            int64_t at = kv0 + n;
            if constexpr (PAGED)
                at = ((int64_t)max(0, min(p.page_table[kv0 + (n >> p.page_shift)], p.num_pages - 1)) << p.page_shift) + (n & ((1 << p.page_shift) - 1));
            const char *vp = p.v + (at * p.ld_v + (int64_t)head * D + d) * S::kSize;
            const float x = BF16 ? __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(vp) << 16) : *reinterpret_cast<const float *>(vp);
            if (!(fabsf(x) < INFINITY)) sum += x;
        }
        if (sum == 0.f) continue;  // (nothing but +-inf or NaN is added)
        if (p.splits > 1) {
            p.part_o[((int64_t)blockIdx.x * S::kRows + e / D) * D + d] += sum;
        } else {
            char *op = p.out + (((tile.q0 + r / p.G) * p.Hq + head * p.G + r % p.G) * (int64_t)D + d) * S::kSize;
            if constexpr (BF16) {
                const float x = __uint_as_float((uint32_t)*reinterpret_cast<uint16_t *>(op) << 16) + sum;
                *reinterpret_cast<uint16_t *>(op) = __builtin_bit_cast(uint16_t, (__bf16)x);
            } else {
                *reinterpret_cast<float *>(op) += sum;
            }
        }
    }
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
    pl.waves = 4;
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
    using S = Shape<BF16, D, 4>;
    const size_t lds = 4 * S::kTileBytes;
    auto *kernel = &prompt_kernel<BF16, D, 4, PAGED>;
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
