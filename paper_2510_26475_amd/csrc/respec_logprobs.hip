// Log-probabilities of given tokens for gfx950, with the entropy of their rows and the best alternatives, and their gradient: what a
// rollout records of the tokens it emits (the log p and log q of Algorithm 1) and what the learner differentiates.
//
// Forward.  One pass over a row: a thread keeps a reference m (a value of the row), s = sum e^{(x-m)/T} and
// t = sum e^{(x-m)/T} (x-m)/T over its pieces, and
//     lse = m/T + ln s,   H = ln s - t/s,   log p(x) = x/T - lse,
// so that neither needs the row's maximum beforehand and the entropy is a difference of small numbers.  The reference is moved only
// where a value lies 2^20 above it.  For the N best logits a wave keeps the maxima of its groups of pieces (128 bytes each, in a
// vocabulary of 151,936): the N groups with the largest ones hold its N best logits, so after the pass those few are read again,
// and the waves' best are ranked by counting, as 64-bit keys of the value in an order-preserving form and the complement of the
// token id.  Bound by HBM (a row is read once); few rows are cut into parts that a second kernel joins in a fixed order.
//
// Gradient.  Reads a row and writes its gradient once, from the lse and H of the forward pass; no statistics.  Bound by HBM.
//
// All sums are fp32 within a thread (some hundred terms), and in a fixed order across threads.
#include "respec_common.hpp"
#include "respec_tiles.hpp"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace respec {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kUnroll = 4;          // pieces in flight per thread
constexpr int kMaxTop = 64;         // alternatives of a row: one per lane
constexpr int kMaxParts = 64;       // parts of a row: one per lane of the wave that joins them
constexpr int kGroups = 640;        // groups of pieces whose maxima a wave keeps
constexpr int kChosen = 64;         // groups of them that are read again
constexpr int kCandidates = 256;    // keys of a wave that are ranked
constexpr int kJoin = 512;          // keys of a row's parts that are ranked
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
    int32_t deep, deep_mul;  // entries of every part's list that the join looks at first; q / deep = q deep_mul / 2^16 for q < 256
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
    int32_t whole_from, whole_to;  // the pieces that lie in the row as a whole
    __device__ Row(const void *logits, int64_t row, int64_t ld, int32_t v) {
        using E = Elem<BF16>;
        base = static_cast<const char *>(logits) + row * ld * E::kSize;
        off = (int32_t)((reinterpret_cast<uintptr_t>(base) & 15) / E::kSize);
        V = v;
        pieces = (int32_t)(((int64_t)off + V + E::kPer - 1) / E::kPer);
        whole_from = off != 0;
        whole_to = (int32_t)(((int64_t)off + V) / E::kPer);
    }
    __device__ int64_t first(int i) const { return (int64_t)i * Elem<BF16>::kPer - off; }
    __device__ bool whole(int i) const { return i >= whole_from && i < whole_to; }
    __device__ const u32x4 *at(int i) const {
        return reinterpret_cast<const u32x4 *>(static_cast<const char *>(base) + first(i) * Elem<BF16>::kSize);
    }
    __device__ int edges() const { return V - max(0, whole_to - whole_from) * Elem<BF16>::kPer; }  // elements in no whole piece
    __device__ int edge(int i) const {  // the i-th of them
        const int head = whole_to > whole_from ? whole_from * Elem<BF16>::kPer - off * (whole_from != 0) : V;
        return i < head ? i : V - edges() + i;
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

// Over the lanes of a wave, in a fixed tree; everybody's result.  `zero` is the operation's neutral value.
template <typename T, typename OP>
__device__ inline T wave_reduce(T x, T zero, OP op) {
    auto from = [&](T y, auto ctrl, auto rows) __attribute__((always_inline)) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, zero), __builtin_bit_cast(int, y), decltype(ctrl)::value,
                                                                 decltype(rows)::value, 0xf, false));
    };
    using std::integral_constant;
    const integral_constant<int, 0xf> all{};
    x = op(x, from(x, integral_constant<int, 0x111>{}, all));                          // row_shr:1
    x = op(x, from(x, integral_constant<int, 0x112>{}, all));                          // row_shr:2
    x = op(x, from(x, integral_constant<int, 0x114>{}, all));                          // row_shr:4
    x = op(x, from(x, integral_constant<int, 0x118>{}, all));                          // row_shr:8
    x = op(x, from(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{}));  // row_bcast:15
    x = op(x, from(x, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{}));  // row_bcast:31
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
__device__ inline uint32_t wave_max(uint32_t x) {
    return wave_reduce(x, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ inline Sums join_wave(Sums a, float scale) {
    const float ref = wave_reduce(a.ref, (float)-INFINITY, [](float x, float y) { return fmaxf(x, y); });
    if (a.ref != ref) move_to(a, ref, scale);
    const auto add = [](float x, float y) { return x + y; };
    return {ref, wave_reduce(a.s, 0.f, add), wave_reduce(a.t, 0.f, add)};
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
    __device__ void start() { list = floor = 0; }
    __device__ void insert(uint64_t key, int top) {
        const int rank = __popcll(__ballot(list > key)), lane = threadIdx.x & 63;
        const uint64_t before = from_lane_before(list);
        list = lane < rank ? list : lane == rank ? key : before;
        floor = read_lane(list, top - 1);
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

__device__ inline uint32_t order_of(float x) { return (uint32_t)(make_key(x, 0) >> 32); }
__device__ inline int bits_below(uint64_t mask) {  // set bits of lanes before this one
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// How the pieces of a part are dealt out: chunks of 64 `deep` pieces, chunk c to wave c % kWaves; an octet of lanes (or a lane, `wide` =
// 1) owns a run of wide * deep pieces of a chunk, its group.
struct Deal {
    int32_t begin, end, deep, wide;
    int32_t chunks;  // of this wave
    __device__ Deal(int b, int e, int wave) : begin(b), end(e) {
        const int per_wave = (e - b + 64 * kWaves - 1) / (64 * kWaves);  // steps of a wave, one piece per lane each
        wide = per_wave <= kGroups / 64 ? 1 : 8;
        deep = wide == 1 ? 1 : (per_wave * 8 + kGroups - 1) / kGroups;
        const int all = (e - b + 64 * deep - 1) / (64 * deep);
        chunks = (all - wave + kWaves - 1) / kWaves;
    }
    __device__ int groups() const { return chunks * (64 / wide); }
    __device__ int piece(int group, int wave, int within) const {  // of a group
        const int chunk = group / (64 / wide), at = group % (64 / wide);
        return begin + ((chunk * kWaves + wave) * 64 + at * wide) * deep + within;
    }
};

// The largest value (in bits from the top down to `last`) that `top` or more of what `reached` counts reach, or a smaller one that exactly
// `top` reach; 0 if there are fewer.  Two bits at a time, as the three counts need not wait for one another.
template <typename F>
__device__ inline uint32_t reached_by(int top, int last, F &&reached) {
    uint32_t least = 0;
    for (int bit = 30; bit >= last; bit -= 2) {
        const uint32_t c1 = least | 1u << bit, c2 = least | 2u << bit, c3 = least | 3u << bit;
        const int n1 = reached(c1), n2 = reached(c2), n3 = reached(c3);
        if (n1 < top) continue;
        least = n3 >= top ? c3 : n2 >= top ? c2 : c1;
        if ((n3 >= top ? n3 : n2 >= top ? n2 : n1) == top) break;
    }
    return least;
}

// The best keys among a wave's groups: the `top` groups with the largest maxima hold them (of groups with equal maxima the first
// ones), so only those, or a few more, are read again.  Leaves them, unsorted and with a few more, in `cand`; returns their number.
template <bool BF16>
__device__ inline int best_of_groups(const Row<BF16> &r, const Deal &deal, int wave, int top, const float *maxima, int32_t *chosen, uint64_t *cand,
                                     int held, float &floor) {
    using E = Elem<BF16>;
    const int lane = threadIdx.x & 63, n = deal.groups();
    uint32_t x[kGroups / 64];  // (0: no group)
#pragma unroll
    for (int j = 0; j < kGroups / 64; ++j) x[j] = j * 64 + lane < n ? order_of(maxima[j * 64 + lane]) : 0u;
    // A value that `top` lanes' own maxima reach: bit by bit, by the upper half alone for bf16, which is all there is to its order.
    constexpr int kLast = BF16 ? 16 : 0;
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < kGroups / 64; ++j) mine = max(mine, x[j]);
    uint32_t least = reached_by(top, kLast, [&](uint32_t from) __attribute__((always_inline)) { return (int)__popcll(__ballot(mine >= from)); });
    auto count = [&](uint32_t from) __attribute__((always_inline)) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < kGroups / 64; ++j)
            if (j * 64 < n) c += (int)__popcll(__ballot(x[j] >= from));
        return c;
    };
    least = max(least, 1u);
    int ties = INT32_MAX, sel = 0;
    if (count(least) > kChosen) {  // Too many groups reach it: the top-th largest maximum of all.
        least = max(reached_by(top, kLast, count), 1u);
        if (count(least) != top) ties = top - count(least + (1u << kLast));
    }
#pragma unroll
    for (int j = 0; j < kGroups / 64; ++j)
        if (j * 64 < n) {
            const bool at = (x[j] ^ least) >> kLast == 0;
            const uint64_t equal = __ballot(at);
            const bool take = x[j] >= least && (!at || bits_below(equal) < ties);
            const uint64_t taken = __ballot(take);
            if (take) chosen[sel + bits_below(taken)] = j * 64 + lane;
            sel += (int)__popcll(taken);
            if (ties != INT32_MAX) ties = max(0, ties - (int)__popcll(equal));
        }
    floor = key_value((uint64_t)least << 32);
    const int run = deal.wide * deal.deep, pieces = sel * run;
    int kept = held;
    for (int q0 = 0; q0 < pieces; q0 += 64) {
        const int q = q0 + lane;
        const int group = run == 1 ? q : q / run;
        const int i = q < pieces ? deal.piece(chosen[group], wave, q - group * run) : deal.end;
        u32x4 raw{};
        if (i < deal.end) raw = *r.at(i);
        float v[E::kPer];
        unpack<BF16>(raw, v);
        const int32_t first = (int32_t)r.first(i);
#pragma unroll
        for (int j = 0; j < E::kPer; ++j) {
            const int32_t e = first + j;
            const bool take = i < deal.end && !(v[j] < floor);
            const uint64_t taken = __ballot(take);
            if (taken == 0) continue;
            const int to = kept + bits_below(taken);
            if (take && to < kCandidates) cand[to] = make_key(v[j], e);
            kept += (int)__popcll(taken);
        }
    }
    if (kept <= kCandidates) return kept;
    // Too many equal ones: one at a time into a sorted list.
    Best best;
    best.start();
    for (int i = 0; i < held; ++i) best.insert(cand[i], top);
    for (int q0 = 0; q0 < pieces; q0 += 64) {
        const int q = q0 + lane;
        const int group = run == 1 ? q : q / run;
        const int i = q < pieces ? deal.piece(chosen[group], wave, q - group * run) : deal.end;
        u32x4 raw{};
        if (i < deal.end) raw = *r.at(i);
        float v[E::kPer];
        unpack<BF16>(raw, v);
        const int32_t first = (int32_t)r.first(i);
        for (int j = 0; j < E::kPer; ++j) {
            const int32_t e = first + j;
            const uint64_t key = i < deal.end ? make_key(v[j], e) : 0;
            uint64_t todo = __ballot(key > best.floor);
            while (todo) {
                best.insert(read_lane(key, __builtin_ctzll(todo)), top);
                todo &= todo - 1;
                todo &= __ballot(key > best.floor);
            }
        }
    }
    if (lane < top) cand[lane] = best.list;
    return top;
}

// One work-group per part of a row.  1,024 rows of 151,936 bf16 logits take 59 us (5.3 TB/s), with 5 alternatives 69: the groups that are read
// again and the ranks come after the pass.  8 rows with 20 alternatives are 64 parts each and take 9.5 us, latency, and 3 to 4.5 for the join.
template <bool BF16, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_kernel(LogprobParams p) {
    using E = Elem<BF16>;
    __shared__ Sums sh_sums[kWaves];
    __shared__ float sh_maxima[TOP ? kWaves * kGroups : 1];
    __shared__ int32_t sh_chosen[TOP ? kWaves * kChosen : 1];
    __shared__ uint64_t sh_cand[TOP ? kWaves * kCandidates : 1];
    __shared__ int sh_kept[kWaves], sh_left;
    __shared__ float sh_floor[kWaves];
    const int row = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int32_t token = p.tokens[row];
    if ((uint32_t)token >= (uint32_t)p.V) {
        if (p.parts == 1) write_unused(p, row);
        return;
    }
    float inv_t;
    const float scale = row_scale_of<BF16>(p, row, inv_t);
    const Row<BF16> r(p.logits, row, p.ld, p.V);
    const float token_logit = load_one<BF16>(r.base, token);
    const int whole = max(0, r.whole_to - r.whole_from);
    const Deal deal(r.whole_from + (int)((int64_t)whole * part / p.parts), r.whole_from + (int)((int64_t)whole * (part + 1) / p.parts), wave);

    Sums a{-INFINITY, 0.f, 0.f};
    int held = 0;
    if (part == 0 && wave == 0) {  // the elements before and behind the whole pieces, one per lane
        held = r.edges();
        if (lane < held) {
            const int e = r.edge(lane);
            const float x = load_one<BF16>(r.base, e);
            if (x > -INFINITY) a = {x, 1.f, 0.f};
            if (!(x < INFINITY)) a.s = NAN;
            if constexpr (TOP) sh_cand[lane] = make_key(x, e);
        }
    }
    float used = a.ref > -INFINITY ? a.ref : 0.f;  // the reference, or 0 while there is none
    float group_max = -INFINITY;
    const float slack = kSlack / scale;
    const int steps = deal.chunks * deal.deep, lane_at = (lane / deal.wide) * deal.wide * deal.deep + lane % deal.wide;
    // (a load in a branch would have to be waited for with all that are on their way, so all lanes load, the last piece if need be)
    int chunk = 0, within = 0;      // of the next step to be requested
    int chunk_at = 0, within_at = 0, done = 0;  // of the next one to be worked on; groups done
    auto request = [&](u32x4(&raw)[kUnroll]) __attribute__((always_inline)) {
        for (int u = 0; u < kUnroll; ++u) {
            const int i = deal.begin + (chunk * kWaves + wave) * 64 * deal.deep + within * deal.wide + lane_at;
            raw[u] = *r.at(min(i, deal.end - 1));
            if (++within == deal.deep) within = 0, chunk = min(chunk + 1, deal.chunks);
        }
    };
    auto work = [&](u32x4(&raw)[kUnroll], int f0) __attribute__((always_inline)) {
        for (int u = 0; u < kUnroll; ++u) {
            if (f0 + u >= steps) break;  // (uniform)
            const int first = deal.begin + (chunk_at * kWaves + wave) * 64 * deal.deep;
            if (first + 64 * deal.deep > deal.end)  // (uniform: the last chunk)
                if (first + within_at * deal.wide + lane_at >= deal.end)
                    for (int w = 0; w < 4; ++w) raw[u][w] = BF16 ? 0xff80ff80u : 0xff800000u;
            float v[E::kPer];
            unpack<BF16>(raw[u], v);
            float largest = v[0];
            for (int j = 1; j < E::kPer; ++j) largest = fmaxf(largest, v[j]);
            if (largest > a.ref + slack || (a.ref == -INFINITY && largest > -INFINITY)) {
                move_to(a, largest, scale);
                used = largest;
            }
            float s = 0.f, t = 0.f;
            // (the difference first: as fma(v, scale, -used * scale) the rounding of that product, half a step of the logit over T, would be in
            // every term, in log p and in the entropy.  1,024 rows of 151,936 take 108.7 us in fp32 this way, 111.6 that way)
            for (int j = 0; j < E::kPer; ++j) {
                const float d = (v[j] - used) * scale, e = __builtin_amdgcn_exp2f(d);
                s += e;
                t += e * fmaxf(d, kFar);
            }
            a.s += s;
            a.t += t;
            if constexpr (TOP) {
                if (deal.wide == 1) {
                    sh_maxima[wave * kGroups + (f0 + u) * 64 + lane] = largest;
                } else {
                    group_max = fmaxf(group_max, largest);
                    if (within_at + 1 == deal.deep) {
                        float m = group_max;  // over the octet: lanes ^ 1, ^ 2, and the mirrored half row
                        m = fmaxf(m, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), 0xb1, 0xf, 0xf, true)));
                        m = fmaxf(m, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), 0x4e, 0xf, 0xf, true)));
                        m = fmaxf(m, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(m), 0x141, 0xf, 0xf, true)));
                        if ((lane & 7) == 0) sh_maxima[wave * kGroups + done * 8 + lane / 8] = m;
                        ++done;
                        group_max = -INFINITY;
                    }
                }
            }
            if (++within_at == deal.deep) within_at = 0, ++chunk_at;
        }
    };
    u32x4 even[kUnroll], odd[kUnroll];  // a batch is worked on while the next one is on its way
    if (steps > 0) request(even);
    for (int f0 = 0; f0 < steps; f0 += 2 * kUnroll) {
        request(odd);
        work(even, f0);
        if (f0 + kUnroll >= steps) break;
        request(even);
        work(odd, f0 + kUnroll);
    }
    a = join_wave(a, scale);
    if (lane == 0) sh_sums[wave] = a;
    if (threadIdx.x == 0) sh_left = 0;
    float floor = -INFINITY;
    if constexpr (TOP) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const int kept = best_of_groups<BF16>(r, deal, wave, p.top, sh_maxima + wave * kGroups, sh_chosen + wave * kChosen, sh_cand + wave * kCandidates, held, floor);
        if (lane == 0) {
            sh_kept[wave] = kept;
            sh_floor[wave] = floor;
        }
    }
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
    if constexpr (TOP) {
        // what the highest of the waves' floors leaves, together; then a key's place is the number of keys above it
        for (int w = 0; w < kWaves; ++w) floor = fmaxf(floor, sh_floor[w]);
        uint64_t *const left = reinterpret_cast<uint64_t *>(sh_maxima);
        static_assert(!TOP || sizeof(sh_maxima) >= sizeof(sh_cand), "room for all");
        for (int c = lane; c < sh_kept[wave]; c += 64) {
            const uint64_t key = sh_cand[wave * kCandidates + c];
            if (key != 0 && !(key_value(key) < floor)) left[atomicAdd(&sh_left, 1)] = key;  // (in any order)
        }
        __syncthreads();
        const int n = sh_left;
        for (int c = threadIdx.x; c < n; c += kThreads) {
            const uint64_t mine = left[c];
            int rank = 0;
#pragma unroll 8
            for (int i = 0; i < n; ++i) rank += left[i] > mine;
            if (rank < p.top) {
                if (p.parts == 1) write_top(p, row, rank, mine, a, inv_t);
                else p.part_top[slot * p.top + rank] = mine;
            }
        }
        if ((int)threadIdx.x < p.top && (int)threadIdx.x >= n) {  // fewer elements than places
            if (p.parts == 1) write_top(p, row, threadIdx.x, 0, a, inv_t);
            else p.part_top[slot * p.top + threadIdx.x] = 0;
        }
    }
}

// Joins the parts of a row.  Sums: a part per lane, in a fixed tree.  Alternatives: the sorted lists' first entries give a value that
// the top-th best is not below, the few keys from there on are ranked by counting.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void logprob_join_kernel(LogprobParams p) {
    extern __shared__ uint64_t keys[];  // [parts][top], then kJoin candidates
    __shared__ int sh_kept;
    __shared__ Sums sh_sums;
    const int row = blockIdx.x, lane = threadIdx.x & 63, top = p.top;
    // (asked for before the token is known: a row without one leaves what is read unused)
    const int64_t slot = (int64_t)row * p.parts;
    const int all = p.parts * top;
    constexpr int kAhead = 8;
    uint64_t early[kAhead] = {};
    if (top > 0)
        for (int j = 0; j < kAhead; ++j) early[j] = p.part_top[slot * top + max(0, min((int)threadIdx.x + j * kThreads, all - 1))];
    Sums a{-INFINITY, 0.f, 0.f};
    if (threadIdx.x < 64 && lane < p.parts) a = {p.part_sums[(slot + lane) * 4], p.part_sums[(slot + lane) * 4 + 1], p.part_sums[(slot + lane) * 4 + 2]};
    const int32_t token = p.tokens[row];
    if ((uint32_t)token >= (uint32_t)p.V) {
        write_unused(p, row);
        return;
    }
    float inv_t;
    const float scale = row_scale_of<BF16>(p, row, inv_t);
    for (int j = 0; j < kAhead; ++j)
        if ((int)threadIdx.x + j * kThreads < all) keys[threadIdx.x + j * kThreads] = early[j];
    for (int i = threadIdx.x + kAhead * kThreads; i < all; i += kThreads) keys[i] = p.part_top[slot * top + i];
    if (threadIdx.x < 64) {
        const float token_logit = load_one<BF16>(static_cast<const char *>(p.logits) + (int64_t)row * p.ld * Elem<BF16>::kSize, token);
        a = join_wave(a, scale);
        if (lane == 0) {
            write_row(p, row, a, token_logit, inv_t);
            sh_sums = a;
            sh_kept = 0;
        }
    }
    if (top == 0) return;
    __syncthreads();
    uint64_t *cand = keys + all;
    // the top-th best of the first `deep` entries of every list, by every wave: of 3 top keys, close to the top-th of all
    // (64 rows with 32 alternatives: 22 us, by a list's first entries alone 34)
    constexpr int kFirsts = 4;
    const int firsts = p.deep * p.parts;
    static_assert(3 * kMaxTop + kMaxParts <= 64 * kFirsts, "a register each");
    uint32_t x[kFirsts] = {};
#pragma unroll
    for (int j = 0; j < kFirsts; ++j)
        if (j * 64 < firsts) {  // (uniform)
            const int q = j * 64 + lane, list = (int)((uint32_t)(q * p.deep_mul) >> 16);
            if (q < firsts) x[j] = (uint32_t)(keys[list * top + q - list * p.deep] >> 32);
        }
    const auto reach = [&](int j, uint32_t from) __attribute__((always_inline)) { return (int)__popcll(__ballot(x[j] >= from)); };
    uint32_t least;
    if (firsts <= 64) least = reached_by(top, BF16 ? 16 : 0, [&](uint32_t from) __attribute__((always_inline)) { return reach(0, from); });
    else least = reached_by(top, BF16 ? 16 : 0, [&](uint32_t from) __attribute__((always_inline)) { return reach(0, from) + reach(1, from) + reach(2, from) + reach(3, from); });
    for (int i = threadIdx.x; i < all; i += kThreads)
        if (keys[i] != 0 && (uint32_t)(keys[i] >> 32) >= least) {
            const int to = atomicAdd(&sh_kept, 1);  // (any order: the ranks are the keys')
            if (to < kJoin) cand[to] = keys[i];
        }
    __syncthreads();
    const int kept = sh_kept;
    a = sh_sums;
    if (kept <= kJoin) {
        for (int c = threadIdx.x; c < kept; c += kThreads) {
            const uint64_t mine = cand[c];
            int rank = 0;
#pragma unroll 8
            for (int i = 0; i < kept; ++i) rank += cand[i] > mine;
            if (rank < top) write_top(p, row, rank, mine, a, inv_t);
        }
        if ((int)threadIdx.x < top && (int)threadIdx.x >= kept) write_top(p, row, threadIdx.x, 0, a, inv_t);
        return;
    }
    // The best keys lie in few lists: the best head of all lists, `top` times.
    if (threadIdx.x >= 64) return;
    uint64_t head = lane < p.parts ? keys[lane * top] : 0, kept_key = 0;
    int next = 1;
    for (int i = 0; i < top; ++i) {
        const uint32_t hi = wave_max((uint32_t)(head >> 32));
        const uint32_t lo = wave_max((uint32_t)(head >> 32) == hi ? (uint32_t)head : 0u);
        const uint64_t key = (uint64_t)hi << 32 | lo;
        if (lane == i) kept_key = key;
        if (key != 0 && head == key) head = next < top ? keys[lane * top + next++] : 0;
    }
    if (lane < top) write_top(p, row, lane, kept_key, a, inv_t);
}

// ------------------------------------------------------------------------------------------ gradient
struct GradRow {
    float inv_t, lse, H, g_lp, g_h;
    int32_t token;
    __device__ float at(float x, int64_t i) const {
        // (log p first: in log2 units the products with 1/T and log2 e of both terms would be rounded before their difference is)
        // (a NaN, of a row that is not finite, stays one in the probability; the maximum would drop it)
        const float log_p = fmaf(x, inv_t, -lse);
        const float prob = __builtin_amdgcn_exp2f(log_p * 1.44269504088896341f);
        float g = -prob * (g_lp + g_h * (fmaxf(log_p, kFar) + H));
        if (i == token) g += g_lp;
        return g * inv_t;
    }
};

// A work-group writes kUnroll * kThreads pieces of a row (or elements, where the two rows lie differently in their 16-byte pieces).
template <bool BF16, bool PIECES>
__global__ __launch_bounds__(kThreads) void logprob_grad_kernel(GradParams p) {
    using E = Elem<BF16>;
    // The last rows first, which the forward pass read last and left in the cache behind the L2s, and loads and stores that take no
    // room there: forward and gradient of 2,048 rows of 151,936 bf16 logits take 300 us; 306 with ordinary loads, 314 with the
    // rows in order as well, 356 with ordinary stores.
    const int row = p.rows - 1 - blockIdx.x / p.blocks_per_row, block = blockIdx.x % p.blocks_per_row;
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
                if (r.whole(i0 + u * kThreads)) raw[u] = __builtin_nontemporal_load(r.at(i0 + u * kThreads));
        for (int u = 0; u < kUnroll; ++u) {
            const int i = i0 + u * kThreads;
            if (i >= r.pieces) break;
            const int64_t first = r.first(i);
            if (r.whole(i)) {
                float v[E::kPer];
                unpack<BF16>(raw[u], v);
                for (int j = 0; j < E::kPer; ++j) v[j] = unused ? 0.f : g.at(v[j], first + j);
                u32x4 w;
                for (int j = 0; j < 4; ++j)
                    w[j] = BF16 ? bf16_bits(v[2 * j]) | bf16_bits(v[(2 * j + 1) % E::kPer]) << 16 : __float_as_uint(v[j]);
                __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(out + first * E::kSize));
            } else {
                for (int64_t e = max(first, (int64_t)0); e < min(first + E::kPer, (int64_t)p.V); ++e)
                    store_one<BF16>(out, e, unused ? 0.f : g.at(load_one<BF16>(r.base, e), e));
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
// Parts of a row: work-groups to fill the device, no part below 256 pieces, and no more parts than a wave has lanes.  Where many alternatives are
// asked for, a wave's part holds three times as many groups, or most of them would be read again (8 rows of 151,936 bf16 logits with
// 64 alternatives take 26 us, in parts of 256 pieces 49).
int parts_of(int32_t rows, int32_t V, int32_t top, bool bf16) {
    const int64_t pieces = V / (bf16 ? 8 : 4);
    const int64_t most = std::min<int64_t>(std::min<int64_t>(kMaxParts, kFill / rows), pieces / std::max(kThreads, 12 * top));
    return (int)std::max<int64_t>(1, most);
}

size_t sums_bytes() { return (size_t)kFill * 4 * sizeof(float); }

template <bool BF16>
void launch_forward(const LogprobParams &p, hipStream_t stream) {
    const dim3 grid((unsigned)((int64_t)p.rows * p.parts));
    if (p.top > 0) hipLaunchKernelGGL((logprob_kernel<BF16, true>), grid, dim3(kThreads), 0, stream, p);
    else hipLaunchKernelGGL((logprob_kernel<BF16, false>), grid, dim3(kThreads), 0, stream, p);
    if (p.parts > 1) hipLaunchKernelGGL((logprob_join_kernel<BF16>), dim3(p.rows), dim3(kThreads), ((size_t)p.parts * p.top + (p.top ? kJoin : 0)) * sizeof(uint64_t), stream, p);
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
    if (!grid_fits(rows, kThreads)) return fail(RESPEC_ERR_UNSUPPORTED, "token_logprobs: too many rows (%d)", rows);
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
    p.parts = parts_of(rows, V, top_n, logits_dt == RESPEC_BF16);
    p.deep = std::max(1, std::min(top_n, (3 * top_n + p.parts - 1) / p.parts));
    p.deep_mul = 65536 / p.deep + 1;
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
    if (!grid_fits(blocks * rows, kThreads)) return fail(RESPEC_ERR_UNSUPPORTED, "token_logprobs_grad: too many rows");
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
