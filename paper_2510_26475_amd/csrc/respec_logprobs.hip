// Log-probabilities of given tokens for gfx950, with the entropy of their rows and the best alternatives, and their gradient: what a
// rollout records of the tokens it emits (the log p and log q of Algorithm 1) and what the learner differentiates.
//
// Forward.  One pass over a row: a thread keeps a reference m (a value of the row), s = sum e^{(x-m)/T} and
// t = sum e^{(x-m)/T} (x-m)/T over its pieces, and
//     lse = m/T + ln s,   H = ln s - t/s,   log p(x) = x/T - lse,
// so that neither needs the row's maximum beforehand and the entropy is a difference of small numbers.  The reference is moved only
// where a value lies 2^20 above it.  The N best logits are kept as 64-bit keys (the value in an order-preserving form, the
// complement of the token id), sorted over the lanes of a wave: a piece whose largest value is below the N-th key costs one
// comparison.  Bound by HBM (a row is read once); few rows are cut into parts that a second kernel joins in a fixed order.
//
// Gradient.  Reads a row and writes its gradient once, from the lse and H of the forward pass; no statistics.  Bound by HBM.
//
// All sums are fp32 within a thread (some hundred terms), and in a fixed order across threads.
#include "respec_common.hpp"

#include <algorithm>
#include <cmath>

namespace respec {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kUnroll = 4;          // pieces in flight per thread
constexpr int kMaxTop = 64;         // alternatives of a row: one per lane
constexpr int kMaxParts = 64;       // parts of a row: one per lane of the wave that joins them
constexpr int kFill = 1024;         // work-groups that a call is cut into where it has fewer rows
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kSlack = 20.f;      // log2 units that a value may lie above its thread's reference
constexpr float kFar = -1000.f;     // (log or log2 units) a weight of zero

struct LogprobParams {
    const void *logits;
    const int32_t *tokens;
    const float *row_temperature;  // [rows] or NULL
    float *logprob, *lse, *entropy;
    int32_t *top_tokens;
    float *top_logprobs;
    int32_t rows, V, top, parts;
    int64_t ld;
    float temperature;
    float *part_sums;    // [rows * parts][4]: reference, s, t
    uint64_t *part_top;  // [rows * parts][top]
};

struct GradParams {
    const void *logits;
    const int32_t *tokens;
    const float *row_temperature;
    const float *lse, *entropy, *grad_logprob, *grad_entropy;
    void *grad;
    int32_t rows, V, blocks_per_row;
    int64_t ld, ld_g;
    float temperature;
};

template <bool BF16>
struct Elem {
    static constexpr int kPer = BF16 ? 8 : 4;  // in a 16-byte piece
    static constexpr int kSize = BF16 ? 2 : 4;
};

template <bool BF16>
__device__ inline float load_one(const void *row, int64_t i) {
    if constexpr (BF16) return __uint_as_float((uint32_t)static_cast<const uint16_t *>(row)[i] << 16);
    else return static_cast<const float *>(row)[i];
}
__device__ inline uint32_t bf16_bits(float x) {  // nearest, ties to even
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}
template <bool BF16>
__device__ inline void store_one(void *row, int64_t i, float x) {
    if constexpr (BF16) static_cast<uint16_t *>(row)[i] = (uint16_t)bf16_bits(x);
    else static_cast<float *>(row)[i] = x;
}
template <bool BF16>
__device__ inline void unpack(u32x4 raw, float *v) {
    if constexpr (BF16) {
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(raw[i] << 16);
            v[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
        }
    } else {
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(raw[i]);
    }
}

// A row as 16-byte pieces counted from the 16-byte border at or before its start: piece i holds the elements
// i * kPer - off ... of the row.
template <bool BF16>
struct Row {
    const void *base;
    int32_t off, V, pieces;
    __device__ Row(const void *logits, int64_t row, int64_t ld, int32_t v) {
        using E = Elem<BF16>;
        base = static_cast<const char *>(logits) + row * ld * E::kSize;
        off = (int32_t)((reinterpret_cast<uintptr_t>(base) & 15) / E::kSize);
        V = v;
        pieces = (int32_t)(((int64_t)off + V + E::kPer - 1) / E::kPer);
    }
    __device__ int64_t first(int i) const { return (int64_t)i * Elem<BF16>::kPer - off; }
    __device__ bool whole(int i) const { return first(i) >= 0 && first(i) + Elem<BF16>::kPer <= V; }
    __device__ const u32x4 *at(int i) const {
        return reinterpret_cast<const u32x4 *>(static_cast<const char *>(base) + first(i) * Elem<BF16>::kSize);
    }
    // The piece's bits; elements outside the row (at its ends) are -inf.
    __device__ u32x4 load(int i) const {
        using E = Elem<BF16>;
        if (whole(i)) return *at(i);
        u32x4 raw;
        for (int w = 0; w < 4; ++w) raw[w] = BF16 ? 0xff80ff80u : 0xff800000u;
        for (int j = 0; j < E::kPer; ++j) {
            const int64_t e = first(i) + j;
            if (e < 0 || e >= V) continue;
            if constexpr (BF16) {
                const uint32_t x = static_cast<const uint16_t *>(base)[e];
                raw[j / 2] = j % 2 ? (raw[j / 2] & 0xffffu) | x << 16 : (raw[j / 2] & 0xffff0000u) | x;
            } else {
                raw[j] = static_cast<const uint32_t *>(base)[e];
            }
        }
        return raw;
    }
};

// Sums of a set of values by their reference (-inf: no value above -inf yet).
struct Sums {
    float ref, s, t;
};
__device__ inline void move_to(Sums &a, float ref, float scale) {
    if (a.ref == -INFINITY) {
        a.ref = ref;  // (s and t are zero, or a NaN that stays)
        return;
    }
    const float d = fmaxf((a.ref - ref) * scale, kFar), f = __builtin_amdgcn_exp2f(d);
    a.t = f * (a.t + a.s * d);
    a.s *= f;
    a.ref = ref;
}
__device__ inline Sums join(Sums a, Sums b, float scale) {
    const float ref = fmaxf(a.ref, b.ref);
    if (a.ref != ref) move_to(a, ref, scale);
    if (b.ref != ref) move_to(b, ref, scale);
    return {ref, a.s + b.s, a.t + b.t};
}

__device__ inline uint64_t make_key(float x, int32_t token) {
    const uint32_t bits = __float_as_uint(x + 0.f);  // (-0 and 0 are equal)
    const uint32_t order = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    return (uint64_t)order << 32 | (uint32_t)~token;
}
__device__ inline float key_value(uint64_t key) {
    const uint32_t order = (uint32_t)(key >> 32);
    return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
__device__ inline int32_t key_token(uint64_t key) { return (int32_t)~(uint32_t)key; }

__device__ inline uint64_t read_lane(uint64_t x, int lane) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, lane), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), lane);
    return (uint64_t)hi << 32 | lo;
}
__device__ inline uint64_t from_lane_before(uint64_t x) {  // (lane 0 keeps its own)
    const uint32_t lo = __builtin_amdgcn_update_dpp((uint32_t)x, (uint32_t)x, 0x138, 0xf, 0xf, false);  // wave_shr:1
    const uint32_t hi = __builtin_amdgcn_update_dpp((uint32_t)(x >> 32), (uint32_t)(x >> 32), 0x138, 0xf, 0xf, false);
    return (uint64_t)hi << 32 | lo;
}

// The best keys of a wave, descending over its lanes; 0 = none.
struct Best {
    uint64_t list, floor;  // floor: the N-th (0 while there are fewer)
    float floor_value;
    int32_t floor_token;
    __device__ void start() {
        list = floor = 0;
        floor_value = -INFINITY;
        floor_token = INT32_MAX;
    }
    __device__ void insert(uint64_t key, int top) {
        const int rank = __popcll(__ballot(list > key)), lane = threadIdx.x & 63;
        const uint64_t before = from_lane_before(list);
        list = lane < rank ? list : lane == rank ? key : before;
        floor = read_lane(list, top - 1);
        if (floor != 0) {
            floor_value = key_value(floor);
            floor_token = key_token(floor);
        }
    }
    // Whether a piece with this largest value, its first element being `first`, can hold a key above the floor.
    __device__ bool may_hold(float largest, int32_t first) const {
        return largest > floor_value || (largest == floor_value && first < floor_token) || floor == 0;
    }
};

template <bool BF16>
__device__ inline float row_scale_of(const LogprobParams &p, int row, float &inv_t) {
    const float T = p.row_temperature ? p.row_temperature[row] : p.temperature;
    inv_t = T >= 1e-30f && T < INFINITY ? 1.f / T : NAN;
    return inv_t * 1.44269504088896341f;
}

// Results of a row, by one thread for its numbers and by `top` threads for its alternatives.
__device__ inline void write_row(const LogprobParams &p, int row, const Sums &a, float token_logit, float inv_t) {
    const float ln_s = logf(a.s);
    p.lse[row] = a.ref * inv_t + ln_s;
    p.logprob[row] = (token_logit - a.ref) * inv_t - ln_s;
    if (p.entropy) p.entropy[row] = ln_s - kLn2 * a.t / a.s;
}
__device__ inline void write_top(const LogprobParams &p, int row, int i, uint64_t key, const Sums &a, float inv_t) {
    const int64_t at = (int64_t)row * p.top + i;
    p.top_tokens[at] = key ? key_token(key) : -1;
    p.top_logprobs[at] = key ? (key_value(key) - a.ref) * inv_t - logf(a.s) : -INFINITY;
}
__device__ inline void write_unused(const LogprobParams &p, int row) {
    if (threadIdx.x == 0) {
        p.logprob[row] = p.lse[row] = 0.f;
        if (p.entropy) p.entropy[row] = 0.f;
    }
    if ((int)threadIdx.x < p.top) {
        p.top_tokens[(int64_t)row * p.top + threadIdx.x] = -1;
        p.top_logprobs[(int64_t)row * p.top + threadIdx.x] = 0.f;
    }
}

// One work-group per part of a row.
template <bool BF16, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_kernel(LogprobParams p) {
    using E = Elem<BF16>;
    __shared__ Sums sh_sums[kWaves];
    __shared__ uint64_t sh_top[TOP ? kWaves * kMaxTop : 1];
    const int row = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int32_t token = p.tokens[row];
    if ((uint32_t)token >= (uint32_t)p.V) {
        if (p.parts == 1) write_unused(p, row);
        return;
    }
    float inv_t;
    const float scale = row_scale_of<BF16>(p, row, inv_t);
    const Row<BF16> r(p.logits, row, p.ld, p.V);
    const float token_logit = load_one<BF16>(r.base, token);
    const int begin = (int)((int64_t)r.pieces * part / p.parts), end = (int)((int64_t)r.pieces * (part + 1) / p.parts);

    Sums a{-INFINITY, 0.f, 0.f};
    float used = 0.f;  // the reference, or 0 while there is none
    Best best;
    if constexpr (TOP) best.start();
    const float slack = kSlack / scale;
    for (int i0 = begin; i0 < end; i0 += kThreads * kUnroll) {
        u32x4 raw[kUnroll];
        for (int u = 0; u < kUnroll; ++u) {
            const int i = i0 + u * kThreads + threadIdx.x;
            if (i < end) raw[u] = r.load(i);
            else
                for (int w = 0; w < 4; ++w) raw[u][w] = BF16 ? 0xff80ff80u : 0xff800000u;
        }
        for (int u = 0; u < kUnroll; ++u) {
            const int i = i0 + u * kThreads + threadIdx.x;
            float v[E::kPer];
            unpack<BF16>(raw[u], v);
            float largest = v[0];
            for (int j = 1; j < E::kPer; ++j) largest = fmaxf(largest, v[j]);
            if (largest > a.ref + slack || (a.ref == -INFINITY && largest > -INFINITY)) {
                move_to(a, largest, scale);
                used = largest;
            }
            float s = 0.f, t = 0.f;
            for (int j = 0; j < E::kPer; ++j) {
                const float d = (v[j] - used) * scale, e = __builtin_amdgcn_exp2f(d);
                s += e;
                t += e * fmaxf(d, kFar);
            }
            a.s += s;
            a.t += t;
            if constexpr (TOP) {
                const int32_t first = (int32_t)r.first(i);
                if (__ballot(i < end && best.may_hold(largest, first)) != 0) {
                    for (int j = 0; j < E::kPer; ++j) {
                        const int32_t e = first + j;
                        const uint64_t key = make_key(v[j], e);
                        uint64_t todo = __ballot(i < end && e >= 0 && e < p.V && key > best.floor);
                        while (todo) {
                            const int from = __builtin_ctzll(todo);
                            best.insert(read_lane(key, from), p.top);
                            todo &= todo - 1;
                            todo &= __ballot(key > best.floor);
                        }
                    }
                }
            }
        }
    }
    for (int step = 1; step < 64; step *= 2) {
        const Sums b{__shfl_xor(a.ref, step), __shfl_xor(a.s, step), __shfl_xor(a.t, step)};
        a = lane & step ? join(b, a, scale) : join(a, b, scale);
    }
    if (lane == 0) sh_sums[wave] = a;
    if constexpr (TOP)
        if (lane < p.top) sh_top[wave * p.top + lane] = best.list;
    __syncthreads();
    a = sh_sums[0];
    for (int w = 1; w < kWaves; ++w) a = join(a, sh_sums[w], scale);
    const int64_t slot = blockIdx.x;
    if (threadIdx.x == 0) {
        if (p.parts == 1) {
            write_row(p, row, a, token_logit, inv_t);
        } else {
            p.part_sums[slot * 4] = a.ref;
            p.part_sums[slot * 4 + 1] = a.s;
            p.part_sums[slot * 4 + 2] = a.t;
        }
    }
    if constexpr (TOP) {  // a key's place is the number of keys above it
        const int n = kWaves * p.top, tid = threadIdx.x;
        int present = 0, rank = 0;
        const uint64_t mine = tid < n ? sh_top[tid] : 0;
        for (int i = 0; i < n; ++i) {
            rank += sh_top[i] > mine;
            present += sh_top[i] != 0;
        }
        if (tid < n && mine != 0 && rank < p.top) {
            if (p.parts == 1) write_top(p, row, rank, mine, a, inv_t);
            else p.part_top[slot * p.top + rank] = mine;
        }
        if (tid < p.top && tid >= present) {
            if (p.parts == 1) write_top(p, row, tid, 0, a, inv_t);
            else p.part_top[slot * p.top + tid] = 0;
        }
    }
}

__device__ inline uint32_t wave_max(uint32_t x) {
    for (int step = 1; step < 64; step *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, step));
    return x;
}

// The parts of a row, one per lane: sums in a fixed tree, alternatives by taking the best head of the sorted lists N times.
template <bool BF16>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobParams p) {
    __shared__ uint64_t sh_top[kMaxTop];
    const int row = blockIdx.x, lane = threadIdx.x;
    const int32_t token = p.tokens[row];
    if ((uint32_t)token >= (uint32_t)p.V) {
        write_unused(p, row);
        return;
    }
    float inv_t;
    const float scale = row_scale_of<BF16>(p, row, inv_t);
    const float token_logit = load_one<BF16>(static_cast<const char *>(p.logits) + (int64_t)row * p.ld * Elem<BF16>::kSize, token);
    const int64_t slot = (int64_t)row * p.parts + lane;
    Sums a{-INFINITY, 0.f, 0.f};
    if (lane < p.parts) a = {p.part_sums[slot * 4], p.part_sums[slot * 4 + 1], p.part_sums[slot * 4 + 2]};
    uint64_t head = 0;
    int next = 1;
    if (p.top > 0 && lane < p.parts) head = p.part_top[slot * p.top];
    for (int step = 1; step < 64; step *= 2) {
        const Sums b{__shfl_xor(a.ref, step), __shfl_xor(a.s, step), __shfl_xor(a.t, step)};
        a = lane & step ? join(b, a, scale) : join(a, b, scale);
    }
    if (lane == 0) write_row(p, row, a, token_logit, inv_t);
    for (int i = 0; i < p.top; ++i) {
        const uint32_t hi = wave_max((uint32_t)(head >> 32));
        const uint32_t lo = wave_max((uint32_t)(head >> 32) == hi ? (uint32_t)head : 0u);
        const uint64_t key = (uint64_t)hi << 32 | lo;
        if (lane == 0) sh_top[i] = key;
        if (key != 0 && head == key) head = next < p.top ? p.part_top[slot * p.top + next++] : 0;
    }
    __syncthreads();
    if (lane < p.top) write_top(p, row, lane, sh_top[lane], a, inv_t);
}

// ------------------------------------------------------------------------------------------ gradient
struct GradRow {
    float inv_t, lse, H, g_lp, g_h;
    int32_t token;
    __device__ float at(float x, int64_t i) const {
        // (log p first: in log2 units the products with 1/T and log2 e of both terms would be rounded before their difference is)
        const float log_p = fmaxf(fmaf(x, inv_t, -lse), kFar);
        const float prob = __builtin_amdgcn_exp2f(log_p * 1.44269504088896341f);
        float g = -prob * (g_lp + g_h * (log_p + H));
        if (i == token) g += g_lp;
        return g * inv_t;
    }
};

// A work-group writes kUnroll * kThreads pieces of a row (or elements, where the two rows lie differently in their 16-byte pieces).
template <bool BF16, bool PIECES>
__global__ __launch_bounds__(kThreads) void logprob_grad_kernel(GradParams p) {
    using E = Elem<BF16>;
    const int row = blockIdx.x / p.blocks_per_row, block = blockIdx.x % p.blocks_per_row;
    const Row<BF16> r(p.logits, row, p.ld, p.V);
    char *out = static_cast<char *>(p.grad) + (int64_t)row * p.ld_g * E::kSize;
    GradRow g;
    g.token = p.tokens[row];
    const bool unused = (uint32_t)g.token >= (uint32_t)p.V;
    const float T = p.row_temperature ? p.row_temperature[row] : p.temperature;
    g.inv_t = T >= 1e-30f && T < INFINITY ? 1.f / T : NAN;
    g.lse = p.lse[row];
    g.g_lp = p.grad_logprob ? p.grad_logprob[row] : 0.f;
    g.g_h = p.grad_entropy ? p.grad_entropy[row] : 0.f;
    g.H = p.grad_entropy ? p.entropy[row] : 0.f;
    if constexpr (PIECES) {
        const int i0 = block * kThreads * kUnroll + threadIdx.x;
        u32x4 raw[kUnroll];
        if (!unused)
            for (int u = 0; u < kUnroll; ++u)
                if (i0 + u * kThreads < r.pieces) raw[u] = r.load(i0 + u * kThreads);
        for (int u = 0; u < kUnroll; ++u) {
            const int i = i0 + u * kThreads;
            if (i >= r.pieces) break;
            const int64_t first = r.first(i);
            float v[E::kPer];
            if (unused)
                for (int j = 0; j < E::kPer; ++j) v[j] = 0.f;
            else {
                unpack<BF16>(raw[u], v);
                for (int j = 0; j < E::kPer; ++j) v[j] = g.at(v[j], first + j);
            }
            if (r.whole(i)) {
                u32x4 w;
                for (int j = 0; j < 4; ++j)
                    w[j] = BF16 ? bf16_bits(v[2 * j]) | bf16_bits(v[(2 * j + 1) % E::kPer]) << 16 : __float_as_uint(v[j]);
                *reinterpret_cast<u32x4 *>(out + first * E::kSize) = w;
            } else {
                for (int j = 0; j < E::kPer; ++j)
                    if (first + j >= 0 && first + j < p.V) store_one<BF16>(out, first + j, v[j]);
            }
        }
    } else {
        for (int u = 0; u < kUnroll * E::kPer; ++u) {
            const int64_t i = ((int64_t)block * kUnroll * E::kPer + u) * kThreads + threadIdx.x;
            if (i < p.V) store_one<BF16>(out, i, unused ? 0.f : g.at(load_one<BF16>(r.base, i), i));
        }
    }
}

// ------------------------------------------------------------------------------------------ host side
// Parts of a row: work-groups to fill the device, no part below 256 pieces, and no more parts than a wave has lanes.
int parts_of(int32_t rows, int32_t V, bool bf16) {
    const int64_t pieces = V / (bf16 ? 8 : 4);
    const int64_t most = std::min<int64_t>(std::min<int64_t>(kMaxParts, kFill / rows), pieces / kThreads);
    return (int)std::max<int64_t>(1, most);
}

size_t sums_bytes() { return (size_t)kFill * 4 * sizeof(float); }

template <bool BF16>
void launch_forward(const LogprobParams &p, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)p.rows * p.parts));
    if (p.top > 0) hipLaunchKernelGGL((logprob_kernel<BF16, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((logprob_kernel<BF16, false>), grid, dim3(kThreads), 0, stream, p);
    if (p.parts > 1) hipLaunchKernelGGL((logprob_join_kernel<BF16>), dim3(p.rows), dim3(64), 0, stream, p);
}

respec_status_t check_rows(const char *name, int32_t rows, int32_t V, int64_t ld, float temperature, bool per_row, respec_dtype_t dt,
                           const void *logits) {
    if (rows <= 0 || V <= 0) return fail(RESPEC_ERR_INVALID_ARG, "%s: need rows > 0 and V > 0 (rows=%d V=%d)", name, rows, V);
    if (dt != RESPEC_F32 && dt != RESPEC_BF16) return fail(RESPEC_ERR_INVALID_ARG, "%s: unknown logits dtype %d", name, (int)dt);
    if (ld < V) return fail(RESPEC_ERR_INVALID_ARG, "%s: row stride smaller than V", name);
    if (!per_row && !(temperature >= 1e-30f && std::isfinite(temperature)))
        return fail(RESPEC_ERR_INVALID_ARG, "%s: temperature must be positive and finite", name);
    if (!aligned_to(logits, dt == RESPEC_BF16 ? 2 : 4)) return fail(RESPEC_ERR_INVALID_ARG, "%s: logits are not aligned to their type", name);
    return RESPEC_OK;
}

}  // namespace
}  // namespace respec

extern "C" {

size_t respec_token_logprobs_workspace_bytes(int32_t rows, int32_t V, int32_t top_n, respec_dtype_t logits_dt) {
    using namespace respec;
    if (rows <= 0 || V <= 0 || top_n < 0 || top_n > kMaxTop || (logits_dt != RESPEC_F32 && logits_dt != RESPEC_BF16)) return 0;
    return round_up(sums_bytes() + (size_t)kFill * top_n * sizeof(uint64_t), 256);
}

respec_status_t respec_token_logprobs(const void *logits, const int32_t *tokens, const float *row_temperature, float *out_logprob,
                                      float *out_lse, float *out_entropy, int32_t *out_top_tokens, float *out_top_logprobs, int32_t rows,
                                      int32_t V, int64_t ld, int32_t top_n, float temperature, respec_dtype_t logits_dt, void *workspace,
                                      size_t workspace_bytes, void *hip_stream) {
    using namespace respec;
    if (!logits || !tokens || !out_logprob || !out_lse) return fail(RESPEC_ERR_INVALID_ARG, "token_logprobs: null pointer argument");
    const respec_status_t st = check_rows("token_logprobs", rows, V, ld, temperature, row_temperature != nullptr, logits_dt, logits);
    if (st != RESPEC_OK) return st;
    if (top_n < 0) return fail(RESPEC_ERR_INVALID_ARG, "token_logprobs: top_n must not be negative (%d)", top_n);
    if (top_n > kMaxTop) return fail(RESPEC_ERR_UNSUPPORTED, "token_logprobs: at most %d alternatives (%d)", kMaxTop, top_n);
    if (top_n > 0 && (!out_top_tokens || !out_top_logprobs))
        return fail(RESPEC_ERR_INVALID_ARG, "token_logprobs: alternatives without a place for them");
    const size_t need = respec_token_logprobs_workspace_bytes(rows, V, top_n, logits_dt);
    if (!workspace || workspace_bytes < need || !aligned_to(workspace, 256))
        return fail(RESPEC_ERR_WORKSPACE, "token_logprobs: workspace of %zu bytes (256-byte aligned) needed, got %zu", need,
                    workspace ? workspace_bytes : (size_t)0);
    LogprobParams p{};
    p.logits = logits;
    p.tokens = tokens;
    p.row_temperature = row_temperature;
    p.logprob = out_logprob;
    p.lse = out_lse;
    p.entropy = out_entropy;
    p.top_tokens = out_top_tokens;
    p.top_logprobs = out_top_logprobs;
    p.rows = rows;
    p.V = V;
    p.top = top_n;
    p.ld = ld;
    p.temperature = temperature;
    p.parts = parts_of(rows, V, logits_dt == RESPEC_BF16);
    p.part_sums = static_cast<float *>(workspace);
    p.part_top = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + sums_bytes());
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (logits_dt == RESPEC_BF16) launch_forward<true>(p, stream);
    else launch_forward<false>(p, stream);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(RESPEC_ERR_HIP, "token_logprobs: launch failed: %s", hipGetErrorString(err));
    clear_error();
    return RESPEC_OK;
}

respec_status_t respec_token_logprobs_grad(const void *logits, const int32_t *tokens, const float *row_temperature, const float *lse,
                                           const float *entropy, const float *grad_logprob, const float *grad_entropy, void *grad_logits,
                                           int32_t rows, int32_t V, int64_t ld, int64_t ld_g, float temperature, respec_dtype_t logits_dt,
                                           void *hip_stream) {
    using namespace respec;
    if (!logits || !tokens || !lse || !grad_logits || (!grad_logprob && !grad_entropy) || (grad_entropy && !entropy))
        return fail(RESPEC_ERR_INVALID_ARG, "token_logprobs_grad: null pointer argument");
    const respec_status_t st = check_rows("token_logprobs_grad", rows, V, ld, temperature, row_temperature != nullptr, logits_dt, logits);
    if (st != RESPEC_OK) return st;
    if (ld_g < V) return fail(RESPEC_ERR_INVALID_ARG, "token_logprobs_grad: row stride smaller than V");
    const bool bf16 = logits_dt == RESPEC_BF16;
    const int64_t esz = bf16 ? 2 : 4;
    if (!aligned_to(grad_logits, (size_t)esz)) return fail(RESPEC_ERR_INVALID_ARG, "token_logprobs_grad: gradient is not aligned to its type");
    GradParams p{};
    p.logits = logits;
    p.tokens = tokens;
    p.row_temperature = row_temperature;
    p.lse = lse;
    p.entropy = entropy;
    p.grad_logprob = grad_logprob;
    p.grad_entropy = grad_entropy;
    p.grad = grad_logits;
    p.rows = rows;
    p.V = V;
    p.ld = ld;
    p.ld_g = ld_g;
    p.temperature = temperature;
    // Whether every row begins at the same place of a 16-byte piece as its gradient's.
    const bool pieces = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(grad_logits)) & 15) == 0 && (ld - ld_g) * esz % 16 == 0;
    const int64_t per_block = (int64_t)kThreads * kUnroll * (bf16 ? 8 : 4);
    const int64_t blocks = (V + (pieces ? 16 / esz - 1 : 0) + per_block - 1) / per_block;
    if (blocks * rows > 0x7fffffff) return fail(RESPEC_ERR_UNSUPPORTED, "token_logprobs_grad: too many rows");
    p.blocks_per_row = (int32_t)blocks;
    const dim3 grid((unsigned)(blocks * rows));
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (bf16 && pieces) hipLaunchKernelGGL((logprob_grad_kernel<true, true>), grid, dim3(kThreads), 0, stream, p);
    else if (bf16) hipLaunchKernelGGL((logprob_grad_kernel<true, false>), grid, dim3(kThreads), 0, stream, p);
    else if (pieces) hipLaunchKernelGGL((logprob_grad_kernel<false, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((logprob_grad_kernel<false, false>), grid, dim3(kThreads), 0, stream, p);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(RESPEC_ERR_HIP, "token_logprobs_grad: launch failed: %s", hipGetErrorString(err));
    clear_error();
    return RESPEC_OK;
}

}  // extern "C"
