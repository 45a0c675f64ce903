// What goes into the paged K/V cache and comes out of it whole: the new tokens' heads normalised, rotated and written in one pass, in the
// cache's type or in 8 bits (respec_quantised.hpp); a cache of 8 bits read back, its accepted tokens committed, its pages copied.  The cache is the one
// that the verify step of Section 2.2 reads and that stays in place while sequences change their kind of decoding (Section 5.2).
#include "respec_common.hpp"
#include "respec_quantised.hpp"
#include "respec_tiles.hpp"

#include <algorithm>
#include <cmath>

namespace respec {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64;

// ------------------------------------------------------------------------------------------ norms, rotation, append
struct WriteParams {
    const char *q, *k, *v;
    char *q_out, *k_pages, *v_pages;
    uint8_t *k_scale, *v_scale;
    const float *q_weight, *k_weight, *inv_freq;
    const int32_t *positions, *q_indptr, *page_indptr, *page_table, *kv_len;
    int64_t ld_q, ld_k, ld_v, ld_out;  // bytes between tokens
    int32_t B, total_q, max_q, num_pages, table_len, page_shift;
    int32_t Hq, Hkv, rotary;           // rotary: rotated entries of a head
    int32_t rows;                      // rows of a work-group: its four waves share them out (1, 2, 4)
    bool interleaved;
    float eps;
};

template <bool BF16>
__device__ inline void unpack(const u32x4 (&raw)[BF16 ? 1 : 2], float (&x)[8]) {
    for (int i = 0; i < 8; ++i)
        x[i] = BF16 ? __uint_as_float(i % 2 ? raw[0][i / 2] & 0xffff0000u : raw[0][i / 2] << 16) : __uint_as_float(raw[BF16 ? 0 : i / 4][i % 4]);
}
template <bool BF16>
__device__ inline void store8(char *to, const float (&x)[8]) {
    if constexpr (BF16) {
        u32x4 w;
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{x[2 * i], x[2 * i + 1]}, bf16x2_t));
        *reinterpret_cast<u32x4 *>(to) = w;
    } else {
        *reinterpret_cast<floatx4 *>(to) = floatx4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<floatx4 *>(to + 16) = floatx4{x[4], x[5], x[6], x[7]};
    }
}

// D / 16 lanes hold a head, each two pieces of eight entries: for pairs (i, i + rotary / 2) a piece and the one with its partners, so that no
// entry leaves its lane but in the sum of squares and the largest magnitude.  A wave goes through the heads of a row, 1024 / D at a time, with the sines
// and cosines of its position worked out once, an angle in each lane (rotary / 2 <= 64 of them: 7.6 us for four rows each of 256 sequences at 28/4 heads,
// 9.2 with eight angles in each of eight lanes' groups).  An angle is position * inv_freq, in turns and in 64 bits until its whole turns are taken off (in
// 32 bits a position of 100,000 would leave an error of 0.004); what 32 bits do not hold of the rest, up to pi 2^-25, is added to its sine and cosine in
// two more products (without them a sine next to its zeros is off by up to 9e-8, many times its rounding; these four rows of 256 sequences take 7.7 us with
// them and 7.6 without).
template <bool BF16, bool E4M3, int D>
__global__ __launch_bounds__(kThreads) void norm_rope_append_kernel(WriteParams p) {
    constexpr int kLanes = D / 16, kHeads = 64 / kLanes;  // lanes of a head, heads of a wave
    constexpr int kSize = BF16 ? 2 : 4, kRaw = BF16 ? 1 : 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane % kLanes, mine = lane / kLanes;
    const int part = wave / p.rows, parts = kWaves / p.rows;
    const int heads = p.Hq + 2 * p.Hkv, units = (heads + kHeads - 1) / kHeads;
    const int64_t token = (int64_t)blockIdx.x * p.rows + wave % p.rows;
    if (token >= p.total_q) return;

    const int pairs = p.interleaved ? 0 : p.rotary / 16;  // pieces whose partners are other pieces
    const int one = p.interleaved ? 2 * c : c < pairs ? c : 2 * c, two = p.interleaved || c >= pairs ? one + 1 : c + pairs;
    const bool turns = 8 * c < p.rotary / 2;  // (whole lanes: rotary is a multiple of 16)

    auto source = [&](int h) __attribute__((always_inline)) {
        const int64_t at = (int64_t)D * kSize;
        return h < p.Hq ? p.q + token * p.ld_q + h * at : h < p.Hq + p.Hkv ? p.k + token * p.ld_k + (h - p.Hq) * at : p.v + token * p.ld_v + (h - p.Hq - p.Hkv) * at;
    };
    u32x4 raw[2][kRaw];
    auto load = [&](int u) __attribute__((always_inline)) {
        const char *from = source(min(u * kHeads + mine, heads - 1));
#pragma unroll
        for (int i = 0; i < kRaw; ++i) {
            raw[0][i] = *reinterpret_cast<const u32x4 *>(from + one * 8 * kSize + i * 16);
            raw[1][i] = *reinterpret_cast<const u32x4 *>(from + two * 8 * kSize + i * 16);
        }
    };
    if (part < units) load(part);  // (on its way while the sequence is looked for)

    // The last sequence that begins at or before the token: 64 places are looked at at a time (four rows each of 256 sequences at
    // 28/4 heads: 9.2 us, and 10.4 with the sequences' rows counted up 64 sequences after the other).
    int b = 0;
    for (int end = p.B; end - b > 1;) {
        const int step = (end - b + 63) / 64, at = b + lane * step;
        const int found = __popcll(__ballot(at < end && p.q_indptr[min(at, end - 1)] <= token));
        b += max(0, found - 1) * step;
        end = min(end, b + step);
    }
    const int q0 = max(0, p.q_indptr[b]), R = max(0, min(p.q_indptr[b + 1], p.total_q)) - q0;
    const int64_t row = token - q0;
    if (row < 0 || row >= min(R, p.max_q)) return;

    // Where K and V go: -1 if the sequence's pages do not have the place.
    const int64_t pos = (int64_t)p.kv_len[b] - R + row;
    int64_t page = -1;
    {
        const int e0 = max(0, min(p.page_indptr[b], p.table_len)), held = max(0, max(0, min(p.page_indptr[b + 1], p.table_len)) - e0);
        if (pos >= 0 && pos < (int64_t)held << p.page_shift) {
            const int32_t id = p.page_table[e0 + (pos >> p.page_shift)];
            if ((uint32_t)id < (uint32_t)p.num_pages) page = id;
        }
    }
    const int slot = (int)(pos & ((1 << p.page_shift) - 1));
    // Sines and cosines: each lane works one angle out, and takes its eight through LDS.
    __shared__ __align__(16) float angles[kWaves][2][64];
    float cs[8], sn[8];
    if (p.rotary > 0) {
        if (2 * lane < p.rotary) {
            const double turn = (double)(p.positions ? (int64_t)p.positions[token] : pos) * 0.15915494309189533577 * (double)p.inv_freq[lane];  // 1 / 2 pi
            const double f = 2.0 * (turn - rint(turn));
            const float lead = (float)f, rest = (float)((f - (double)lead) * 3.14159265358979323846);  // (half turns; radians)
            float s0, c0;
            sincospif(lead, &s0, &c0);
            angles[wave][0][lane] = fmaf(c0, rest, s0);
            angles[wave][1][lane] = fmaf(-s0, rest, c0);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (turns)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sn[j] = angles[wave][0][8 * c + j];
                cs[j] = angles[wave][1][8 * c + j];
            }
    }

    for (int u = part; u < units; u += parts) {
        const int h = u * kHeads + mine;
        const bool is_q = h < p.Hq, is_k = !is_q && h < p.Hq + p.Hkv;
        float x[2][8];
        unpack<BF16>(raw[0], x[0]);
        unpack<BF16>(raw[1], x[1]);
        if (u + parts < units) load(u + parts);
        const float *weight = is_q ? p.q_weight : is_k ? p.k_weight : nullptr;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(x[i / 8][i % 8], x[i / 8][i % 8], sum);
#pragma unroll
        for (int step = 1; step < kLanes; step *= 2) sum += __shfl_xor(sum, step);
        if (weight) {
            const float r = 1.f / sqrtf(sum * (1.f / D) + p.eps);
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const floatx4 w = *reinterpret_cast<const floatx4 *>(weight + (i < 8 ? one : two) * 8 + i % 8);
                for (int j = 0; j < 4; ++j) x[i / 8][i % 8 + j] *= r * w[j];
            }
        }
        if (turns && (is_q || is_k)) {
            auto turn = [&](float &e, float &f, int j) __attribute__((always_inline)) {
                const float e0 = e, f0 = f;
                e = e0 * cs[j] - f0 * sn[j];
                f = f0 * cs[j] + e0 * sn[j];
            };
            if (p.interleaved) {
#pragma unroll
                for (int j = 0; j < 8; ++j) turn(x[j / 4][j % 4 * 2], x[j / 4][j % 4 * 2 + 1], j);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) turn(x[0][j], x[1][j], j);
            }
        }
        float top = 0.f;
        if constexpr (E4M3) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float y = fabsf(x[i / 8][i % 8]);
                top = fmaxf(top, y < INFINITY ? y : 0.f);
            }
#pragma unroll
            for (int step = 1; step < kLanes; step *= 2) top = fmaxf(top, __shfl_xor(top, step));
        }
        if (h >= heads) continue;
        if (is_q) {
            char *to = p.q_out + token * p.ld_out + (int64_t)h * D * kSize;
            store8<BF16>(to + one * 8 * kSize, x[0]);
            store8<BF16>(to + two * 8 * kSize, x[1]);
        } else if (page >= 0) {
            const int head = is_k ? h - p.Hq : h - p.Hq - p.Hkv;
            char *const pool = is_k ? p.k_pages : p.v_pages;
            const int64_t at = (((page << p.page_shift) + slot) * p.Hkv + head) * D;
            if constexpr (E4M3) {
                const int byte = scale_byte(top);
                const float inv = inverse_of(byte);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float lo[4] = {x[i][0] * inv, x[i][1] * inv, x[i][2] * inv, x[i][3] * inv};
                    const float hi[4] = {x[i][4] * inv, x[i][5] * inv, x[i][6] * inv, x[i][7] * inv};
                    *reinterpret_cast<u32x2 *>(pool + at + (i ? two : one) * 8) = u32x2{codes_of(lo), codes_of(hi)};
                }
                if (c == 0) (is_k ? p.k_scale : p.v_scale)[((page * p.Hkv + head) << p.page_shift) + slot] = (uint8_t)byte;
            } else {
                store8<BF16>(pool + (at + one * 8) * kSize, x[0]);
                store8<BF16>(pool + (at + two * 8) * kSize, x[1]);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ a cache of 8 bits: read back, commit, copy
struct ReadParams {
    const char *k, *v;
    const uint8_t *k_scale, *v_scale;
    const int32_t *page_indptr, *page_table, *kv_len;
    const int64_t *kv_indptr;
    char *k_out, *v_out;
    int64_t total_kv;
    int32_t B, max_kv, num_pages, table_len, page_shift, Hkv, pieces;  // pieces: of 16 codes in a head
};
constexpr int kReadRows = 16;  // of a work-group

// A thread turns 16 codes of K and of V of a token into 32 (fp32: 64) bytes each.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void read_quantised_kernel(ReadParams p) {
    const int64_t row0 = (int64_t)blockIdx.x * kReadRows;
    int first = 0;
    for (int end = p.B; end - first > 1;) {  // the last sequence that begins at or before row0
        const int at = (first + end) / 2;
        if (p.kv_indptr[at] <= row0) first = at;
        else end = at;
    }
    const int per_row = p.Hkv * p.pieces;
    for (int i = threadIdx.x; i < kReadRows * per_row; i += kThreads) {
        const int64_t row = row0 + i / per_row;
        if (row >= p.total_kv) break;
        const int rest = i % per_row, head = rest / p.pieces, piece = rest % p.pieces;
        int b = first;
        while (b + 1 < p.B && p.kv_indptr[b + 1] <= row) ++b;
        const int64_t j = row - p.kv_indptr[b];
        if (j < 0 || row >= p.kv_indptr[b + 1]) continue;
        const int e0 = max(0, min(p.page_indptr[b], p.table_len)), held = max(0, max(0, min(p.page_indptr[b + 1], p.table_len)) - e0);
        if (j >= min(p.kv_len[b], p.max_kv) || j >= (int64_t)held << p.page_shift) continue;
        const int32_t id = p.page_table[e0 + (j >> p.page_shift)];
        if ((uint32_t)id >= (uint32_t)p.num_pages) continue;
        const int slot = (int)(j & ((1 << p.page_shift) - 1));
        const int64_t from = ((((int64_t)id << p.page_shift) + slot) * p.Hkv + head) * p.pieces + piece, scale = (((int64_t)id * p.Hkv + head) << p.page_shift) + slot;
        const int64_t to = (row * p.Hkv + head) * p.pieces + piece;
        const u32x4 kc = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p.k) + from), vc = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p.v) + from);
        const float ks = scale_of(p.k_scale[scale]), vs = scale_of(p.v_scale[scale]);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const u32x4 codes = w ? vc : kc;
            const float step = w ? vs : ks;
            char *out = (w ? p.v_out : p.k_out) + to * (BF16 ? 32 : 64);
            if constexpr (BF16) {
                uint32_t x[8];
#pragma unroll
                for (int y = 0; y < 4; ++y) values_of(codes[y], step, x[2 * y], x[2 * y + 1]);
                *reinterpret_cast<u32x4 *>(out) = u32x4{x[0], x[1], x[2], x[3]};
                *reinterpret_cast<u32x4 *>(out + 16) = u32x4{x[4], x[5], x[6], x[7]};
            } else {
#pragma unroll
                for (int y = 0; y < 4; ++y) *reinterpret_cast<floatx4 *>(out + 16 * y) = floats_of(codes[y], step);
            }
        }
    }
}

struct CommitQParams {
    char *k, *v;
    uint8_t *k_scale, *v_scale;
    const int32_t *q_indptr, *page_indptr, *page_table, *path, *num_accepted;
    int32_t *kv_len;
    int32_t B, total_q, max_q, num_pages, table_len, page_shift, path_stride, Hkv, token_bytes;
};

// As the commit of the other types, codes and scales: a work-group per sequence.  A thread always handles the same pieces and the same heads' scales, and a
// later move never reads what an earlier one wrote over (rows increase along the path), so program order is enough.
__global__ __launch_bounds__(kThreads) void commit_quantised_kernel(CommitQParams p) {
    const int b = blockIdx.x;
    const int q0 = max(0, min(p.q_indptr[b], p.total_q));
    const int R = max(0, min(max(0, min(p.q_indptr[b + 1], p.total_q)) - q0, p.max_q));
    const int e0 = max(0, min(p.page_indptr[b], p.table_len)), held = max(0, max(0, min(p.page_indptr[b + 1], p.table_len)) - e0);
    __shared__ int sh_len;  // (read by the thread that overwrites it: a wave that starts late must not see the new length)
    if (threadIdx.x == 0) sh_len = p.kv_len[b];
    __syncthreads();
    const int64_t L = max((int64_t)0, min((int64_t)sh_len, (int64_t)held << p.page_shift));
    if (R < 1 || L < R) return;
    const int first_new = (int)(L - R);
    int n = max(0, min(p.num_accepted[b], R - 1));
    if (p.path) n = min(n, p.path_stride);
    auto page_of = [&](int pos) __attribute__((always_inline)) -> int64_t { return max(0, min(p.page_table[e0 + (pos >> p.page_shift)], p.num_pages - 1)); };
    const int mask = (1 << p.page_shift) - 1;
    int done = 0;
    for (int j = 0; j < n; ++j) {
        const int r = p.path ? p.path[(int64_t)b * p.path_stride + j] : j + 1;
        if (r < j + 1 || r >= R) break;
        done = j + 1;
        if (r == j + 1) continue;
        const int from = first_new + r, to = first_new + 1 + j;
        const int64_t src = page_of(from), dst = page_of(to);
        for (int i = threadIdx.x; i < p.token_bytes / 16; i += kThreads) {
            const int64_t s = ((src << p.page_shift) + (from & mask)) * p.token_bytes + (int64_t)i * 16, d = ((dst << p.page_shift) + (to & mask)) * p.token_bytes + (int64_t)i * 16;
            const u32x4 x = *reinterpret_cast<const u32x4 *>(p.k + s), y = *reinterpret_cast<const u32x4 *>(p.v + s);
            *reinterpret_cast<u32x4 *>(p.k + d) = x;
            *reinterpret_cast<u32x4 *>(p.v + d) = y;
        }
        for (int h = threadIdx.x; h < p.Hkv; h += kThreads) {
            const int64_t s = ((src * p.Hkv + h) << p.page_shift) + (from & mask), d = ((dst * p.Hkv + h) << p.page_shift) + (to & mask);
            const uint8_t x = p.k_scale[s], y = p.v_scale[s];
            p.k_scale[d] = x;
            p.v_scale[d] = y;
        }
    }
    if (threadIdx.x == 0) p.kv_len[b] = first_new + 1 + done;
}

struct CopyQParams {
    char *pool[4];          // codes of K and V, scales of K and V
    const int32_t *src, *dst;
    int64_t page_bytes[2];  // of codes, of scales
    int32_t n, num_pages, chunks[2];
};
constexpr int kChunk = kThreads * 16 * 4;  // bytes of a page that a work-group moves at a time

__global__ __launch_bounds__(kThreads) void copy_quantised_kernel(CopyQParams p) {
    const int per_page = 2 * (p.chunks[0] + p.chunks[1]);
    const int64_t items = (int64_t)p.n * per_page;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const int i = (int)(it / per_page), rest = (int)(it % per_page);
        const int scales = rest >= 2 * p.chunks[0], at_piece = (scales ? rest - 2 * p.chunks[0] : rest) >> 1;
        const int32_t src = p.src[i], dst = p.dst[i];
        if ((uint32_t)src >= (uint32_t)p.num_pages || (uint32_t)dst >= (uint32_t)p.num_pages || src == dst) continue;
        const int64_t bytes = scales ? p.page_bytes[1] : p.page_bytes[0], at = (int64_t)at_piece * kChunk;
        char *const pool = scales ? (rest & 1 ? p.pool[3] : p.pool[2]) : (rest & 1 ? p.pool[1] : p.pool[0]);
        u32x4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t o = at + ((int64_t)j * kThreads + threadIdx.x) * 16;
            if (o < bytes) x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(pool + src * bytes + o));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t o = at + ((int64_t)j * kThreads + threadIdx.x) * 16;
            if (o < bytes) __builtin_nontemporal_store(x[j], reinterpret_cast<u32x4 *>(pool + dst * bytes + o));
        }
    }
}

// ------------------------------------------------------------------------------------------ host side
int shift_of(int32_t page_size) {
    if (page_size < 16 || page_size > 1024 || (page_size & (page_size - 1)) != 0) return -1;
    return __builtin_ctz((unsigned)page_size);
}

respec_status_t launched(const char *name) {
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(RESPEC_ERR_HIP, "%s: launch failed: %s", name, hipGetErrorString(err));
    clear_error();
    return RESPEC_OK;
}

// What the calls on pools of 8 bits have in common.
respec_status_t check_pools(const char *name, const void *k, const void *v, const void *ks, const void *vs, int32_t num_pages, int32_t page_size, int32_t Hkv,
                            int32_t D) {
    if (!k || !v || !ks || !vs) return fail(RESPEC_ERR_INVALID_ARG, "%s: null pointer argument", name);
    if (num_pages <= 0 || Hkv <= 0 || D <= 0) return fail(RESPEC_ERR_INVALID_ARG, "%s: sizes must be positive (num_pages=%d Hkv=%d D=%d)", name, num_pages, Hkv, D);
    if (shift_of(page_size) < 0) return fail(RESPEC_ERR_UNSUPPORTED, "%s: page size %d is not a power of two in [16, 1024]", name, page_size);
    if (D != 64 && D != 128) return fail(RESPEC_ERR_UNSUPPORTED, "%s: head size %d is neither 64 nor 128", name, D);
    if ((int64_t)Hkv * D > (1 << 24)) return fail(RESPEC_ERR_UNSUPPORTED, "%s: Hkv*D must be at most 2^24", name);
    if (!aligned_to(k, 16) || !aligned_to(v, 16) || !aligned_to(ks, 16) || !aligned_to(vs, 16))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: pools and scales must be 16-byte aligned", name);
    return RESPEC_OK;
}

template <bool BF16, bool E4M3>
void launch_write(const WriteParams &p, int32_t D, unsigned grid, hipStream_t stream) {
    if (D == 128) hipLaunchKernelGGL((norm_rope_append_kernel<BF16, E4M3, 128>), dim3(grid), dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((norm_rope_append_kernel<BF16, E4M3, 64>), dim3(grid), dim3(kThreads), 0, stream, p);
}

}  // namespace
}  // namespace respec

extern "C" {

respec_status_t respec_norm_rope_append_paged(const void *q, const void *k, const void *v, const float *q_weight, const float *k_weight,
                                              const float *inv_freq, const int32_t *positions, void *q_out, void *k_pages, void *v_pages,
                                              uint8_t *k_scale, uint8_t *v_scale, const int32_t *q_indptr, const int32_t *page_indptr,
                                              const int32_t *page_table, const int32_t *kv_len, int32_t B, int32_t total_q, int32_t max_q_per_seq,
                                              int32_t num_pages, int32_t page_table_len, int32_t page_size, int32_t Hq, int32_t Hkv, int32_t D,
                                              int32_t rotary_dim, int32_t interleaved, int64_t ld_q, int64_t ld_k, int64_t ld_v, int64_t ld_q_out, float eps,
                                              respec_dtype_t dt, respec_dtype_t pool_dt, void *hip_stream) {
    using namespace respec;
    static const char *name = "norm_rope_append_paged";
    if (!k || !v || !k_pages || !v_pages || !q_indptr || !page_indptr || !page_table || !kv_len || !q != !q_out || (!q && q_weight))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: null pointer argument (q, q_out and q_weight go together)", name);
    if (B <= 0 || total_q <= 0 || max_q_per_seq <= 0 || num_pages <= 0 || page_table_len <= 0 || Hq <= 0 || Hkv <= 0 || D <= 0)
        return fail(RESPEC_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d total_q=%d max_q=%d Hq=%d Hkv=%d)", name, B, total_q, max_q_per_seq, Hq, Hkv);
    if ((dt != RESPEC_F32 && dt != RESPEC_BF16) || (pool_dt != dt && pool_dt != RESPEC_E4M3))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: types %d and %d of the heads and of the pools", name, (int)dt, (int)pool_dt);
    if ((pool_dt == RESPEC_E4M3) != (k_scale != nullptr) || !k_scale != !v_scale)
        return fail(RESPEC_ERR_INVALID_ARG, "%s: k_scale and v_scale belong to pools of 8 bits, and only to them", name);
    if (D != 64 && D != 128) return fail(RESPEC_ERR_UNSUPPORTED, "%s: head size %d is neither 64 nor 128", name, D);
    if (rotary_dim < 0 || rotary_dim > D || !inv_freq != (rotary_dim == 0))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: rotary_dim=%d must lie in [0, D], and be 0 without inv_freq", name, rotary_dim);
    if (rotary_dim % 16 != 0) return fail(RESPEC_ERR_UNSUPPORTED, "%s: rotary_dim=%d is not a multiple of 16", name, rotary_dim);
    if (!std::isfinite(eps) || eps < 0.f) return fail(RESPEC_ERR_INVALID_ARG, "%s: eps must be finite and not negative", name);
    const int shift = shift_of(page_size);
    if (shift < 0) return fail(RESPEC_ERR_UNSUPPORTED, "%s: page size %d is not a power of two in [16, 1024]", name, page_size);
    const int64_t esz = dt == RESPEC_BF16 ? 2 : 4;
    if ((int64_t)Hkv * D * esz > (1 << 24) || (int64_t)Hq * D * esz > (1 << 24)) return fail(RESPEC_ERR_UNSUPPORTED, "%s: a token's heads take more than 2^24 bytes", name);
    if (ld_k < (int64_t)Hkv * D || ld_v < (int64_t)Hkv * D || (q && (ld_q < (int64_t)Hq * D || ld_q_out < (int64_t)Hq * D)))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: a token stride is smaller than a token", name);
    if (ld_k * esz % 16 != 0 || ld_v * esz % 16 != 0 || (q && (ld_q * esz % 16 != 0 || ld_q_out * esz % 16 != 0)))
        return fail(RESPEC_ERR_UNSUPPORTED, "%s: token strides must be multiples of 16 bytes", name);
    for (const void *x : {q, k, v, static_cast<const void *>(q_out), static_cast<const void *>(k_pages), static_cast<const void *>(v_pages),
                          static_cast<const void *>(q_weight), static_cast<const void *>(k_weight), static_cast<const void *>(k_scale), static_cast<const void *>(v_scale)})
        if (!aligned_to(x, 16)) return fail(RESPEC_ERR_INVALID_ARG, "%s: data pointers and scales must be 16-byte aligned", name);
    WriteParams p{};
    p.q = static_cast<const char *>(q);
    p.k = static_cast<const char *>(k);
    p.v = static_cast<const char *>(v);
    p.q_out = static_cast<char *>(q_out);
    p.k_pages = static_cast<char *>(k_pages);
    p.v_pages = static_cast<char *>(v_pages);
    p.k_scale = k_scale;
    p.v_scale = v_scale;
    p.q_weight = q_weight;
    p.k_weight = k_weight;
    p.inv_freq = inv_freq;
    p.positions = positions;
    p.q_indptr = q_indptr;
    p.page_indptr = page_indptr;
    p.page_table = page_table;
    p.kv_len = kv_len;
    p.ld_q = ld_q * esz;
    p.ld_k = ld_k * esz;
    p.ld_v = ld_v * esz;
    p.ld_out = ld_q_out * esz;
    p.B = B;
    p.total_q = total_q;
    p.max_q = max_q_per_seq;
    p.num_pages = num_pages;
    p.table_len = page_table_len;
    p.page_shift = shift;
    p.Hq = q ? Hq : 0;
    p.Hkv = Hkv;
    p.rotary = rotary_dim;
    p.interleaved = interleaved != 0;
    p.eps = eps;
    // Few rows: four waves share one row's heads; many: each has a row of its own, and looks one position's angles up for all its heads.  28/4 heads in bf16, one row
    // and four to a work-group: 256 rows 4.6 and 6.8 us, 1,024 6.8 and 7.9, 2,048 11.4 and 10.6, 4,096 19.3 and 15.5 (the two cross between 1,000 and 2,000 rows
    // for 16/2 and 40/8 heads and over 8 bits too).
    p.rows = total_q <= 2048 ? 1 : 4;
    const int64_t grid = ((int64_t)total_q + p.rows - 1) / p.rows;
    if (!grid_fits(grid, kThreads)) return fail(RESPEC_ERR_UNSUPPORTED, "%s: too many rows", name);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dt == RESPEC_BF16) pool_dt == RESPEC_E4M3 ? launch_write<true, true>(p, D, (unsigned)grid, stream) : launch_write<true, false>(p, D, (unsigned)grid, stream);
    else pool_dt == RESPEC_E4M3 ? launch_write<false, true>(p, D, (unsigned)grid, stream) : launch_write<false, false>(p, D, (unsigned)grid, stream);
    return launched(name);
}

respec_status_t respec_read_paged_quantised(const void *k_pages, const void *v_pages, const uint8_t *k_scale, const uint8_t *v_scale,
                                            const int32_t *page_indptr, const int32_t *page_table, const int32_t *kv_len, const int64_t *kv_indptr,
                                            void *k_out, void *v_out, int32_t B, int64_t total_kv, int32_t max_kv_len, int32_t num_pages,
                                            int32_t page_table_len, int32_t page_size, int32_t Hkv, int32_t D, respec_dtype_t dt, void *hip_stream) {
    using namespace respec;
    static const char *name = "read_paged_quantised";
    const respec_status_t st = check_pools(name, k_pages, v_pages, k_scale, v_scale, num_pages, page_size, Hkv, D);
    if (st != RESPEC_OK) return st;
    if (!page_indptr || !page_table || !kv_len || !kv_indptr || !k_out || !v_out) return fail(RESPEC_ERR_INVALID_ARG, "%s: null pointer argument", name);
    if (B <= 0 || total_kv <= 0 || max_kv_len <= 0 || page_table_len <= 0)
        return fail(RESPEC_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d total_kv=%lld max_kv=%d)", name, B, (long long)total_kv, max_kv_len);
    if (dt != RESPEC_F32 && dt != RESPEC_BF16) return fail(RESPEC_ERR_INVALID_ARG, "%s: unknown dtype %d", name, (int)dt);
    if (!aligned_to(k_out, 16) || !aligned_to(v_out, 16)) return fail(RESPEC_ERR_INVALID_ARG, "%s: data pointers must be 16-byte aligned", name);
    const int64_t grid = total_kv / kReadRows + (total_kv % kReadRows != 0);
    if (!grid_fits(grid, kThreads)) return fail(RESPEC_ERR_UNSUPPORTED, "%s: too many tokens", name);
    ReadParams p{};
    p.k = static_cast<const char *>(k_pages);
    p.v = static_cast<const char *>(v_pages);
    p.k_scale = k_scale;
    p.v_scale = v_scale;
    p.page_indptr = page_indptr;
    p.page_table = page_table;
    p.kv_len = kv_len;
    p.kv_indptr = kv_indptr;
    p.k_out = static_cast<char *>(k_out);
    p.v_out = static_cast<char *>(v_out);
    p.total_kv = total_kv;
    p.B = B;
    p.max_kv = max_kv_len;
    p.num_pages = num_pages;
    p.table_len = page_table_len;
    p.page_shift = shift_of(page_size);
    p.Hkv = Hkv;
    p.pieces = D / 16;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dt == RESPEC_BF16) hipLaunchKernelGGL(read_quantised_kernel<true>, dim3((unsigned)grid), dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL(read_quantised_kernel<false>, dim3((unsigned)grid), dim3(kThreads), 0, stream, p);
    return launched(name);
}

respec_status_t respec_commit_accepted_paged_quantised(void *k_pages, void *v_pages, uint8_t *k_scale, uint8_t *v_scale, const int32_t *q_indptr,
                                                       const int32_t *page_indptr, const int32_t *page_table, int32_t *kv_len, const int32_t *path,
                                                       int32_t path_stride, const int32_t *num_accepted, int32_t B, int32_t total_q,
                                                       int32_t max_q_per_seq, int32_t num_pages, int32_t page_table_len, int32_t page_size, int32_t Hkv,
                                                       int32_t D, void *hip_stream) {
    using namespace respec;
    static const char *name = "commit_accepted_paged_quantised";
    const respec_status_t st = check_pools(name, k_pages, v_pages, k_scale, v_scale, num_pages, page_size, Hkv, D);
    if (st != RESPEC_OK) return st;
    if (!q_indptr || !page_indptr || !page_table || !kv_len || !num_accepted) return fail(RESPEC_ERR_INVALID_ARG, "%s: null pointer argument", name);
    if (B <= 0 || total_q <= 0 || max_q_per_seq <= 0 || page_table_len <= 0 || (path && path_stride <= 0))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: sizes must be positive (B=%d total_q=%d max_q=%d)", name, B, total_q, max_q_per_seq);
    if (!grid_fits(B, kThreads)) return fail(RESPEC_ERR_UNSUPPORTED, "%s: too many sequences (%d)", name, B);
    CommitQParams p{};
    p.k = static_cast<char *>(k_pages);
    p.v = static_cast<char *>(v_pages);
    p.k_scale = k_scale;
    p.v_scale = v_scale;
    p.q_indptr = q_indptr;
    p.page_indptr = page_indptr;
    p.page_table = page_table;
    p.path = path;
    p.num_accepted = num_accepted;
    p.kv_len = kv_len;
    p.B = B;
    p.total_q = total_q;
    p.max_q = max_q_per_seq;
    p.num_pages = num_pages;
    p.table_len = page_table_len;
    p.page_shift = shift_of(page_size);
    p.path_stride = path_stride;
    p.Hkv = Hkv;
    p.token_bytes = Hkv * D;
    hipLaunchKernelGGL(commit_quantised_kernel, dim3((unsigned)B), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
    return launched(name);
}

respec_status_t respec_pages_copy_quantised(void *k_pages, void *v_pages, uint8_t *k_scale, uint8_t *v_scale, const int32_t *copy_src,
                                            const int32_t *copy_dst, int32_t n, int32_t num_pages, int32_t page_size, int32_t Hkv, int32_t D,
                                            void *hip_stream) {
    using namespace respec;
    static const char *name = "pages_copy_quantised";
    const respec_status_t st = check_pools(name, k_pages, v_pages, k_scale, v_scale, num_pages, page_size, Hkv, D);
    if (st != RESPEC_OK) return st;
    if (!copy_src || !copy_dst) return fail(RESPEC_ERR_INVALID_ARG, "%s: null pointer argument", name);
    if (n <= 0) return fail(RESPEC_ERR_INVALID_ARG, "%s: sizes must be positive (n=%d)", name, n);
    CopyQParams p{};
    p.pool[0] = static_cast<char *>(k_pages);
    p.pool[1] = static_cast<char *>(v_pages);
    p.pool[2] = reinterpret_cast<char *>(k_scale);
    p.pool[3] = reinterpret_cast<char *>(v_scale);
    p.src = copy_src;
    p.dst = copy_dst;
    p.page_bytes[1] = (int64_t)Hkv * page_size;
    p.page_bytes[0] = p.page_bytes[1] * D;
    for (int i = 0; i < 2; ++i) p.chunks[i] = (int32_t)((p.page_bytes[i] + kChunk - 1) / kChunk);
    p.n = n;
    p.num_pages = num_pages;
    const int64_t items = (int64_t)n * 2 * (p.chunks[0] + p.chunks[1]);
    hipLaunchKernelGGL(copy_quantised_kernel, dim3((unsigned)std::min<int64_t>(items, 4096)), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
    return launched(name);
}

}  // extern "C"
