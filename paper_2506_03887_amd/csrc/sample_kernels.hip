// gfx950 kernels of the sampler behind the mask: one token a row by temperature, top-k, top-p and min-p, from one given random
// number a row.  The logits are read, nothing is written back.
//
// The order of the draw is that of the logits, descending, equal ones by ascending id; w = exp((l - max) / temperature).  Top-k,
// top-p and min-p each keep a prefix of that order, so what is drawn from is its first n tokens, and everything that has to be found
// is a place in the order: the token number n, or the token at which the summed weights pass a border.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "argmax.hpp"
#include "launch.hpp"
#include "stream_access.hpp"

namespace pre3 {

namespace {

constexpr int kSampleBlock = 1024, kSampleWaves = kSampleBlock / 64;

// What a row is drawn by.  A temperature that is not above zero decodes greedily (the draw from one token).
struct RowDraw {
    double rate, top_p, min_p, uniform;      // rate: 1 / temperature; top_p 1 and min_p 0: off
    int top_k;                               // 0: off
};
__device__ __forceinline__ RowDraw row_draw(const SampleRows &rows, int b) {
    RowDraw d;
    const float t = rows.temperature ? rows.temperature[b] : 1.0f, u = rows.uniform[b];
    const float p = rows.top_p ? rows.top_p[b] : 1.0f, m = rows.min_p ? rows.min_p[b] : 0.0f;
    const int k = rows.top_k ? rows.top_k[b] : 0;
    const bool greedy = !(t > 0.0f);
    d.rate = greedy ? 1.0 : 1.0 / (double)t;
    d.top_k = greedy ? 1 : k > 0 ? k : 0;
    d.top_p = p < 1.0f ? (double)p : 1.0;    // (a NaN is off)
    d.min_p = m > 0.0f ? (double)m : 0.0;
    d.uniform = u > 0.0f ? (u < 1.0f ? (double)u : 1.0) : 0.0;
    return d;
}
// e^x for x <= 0 in 64 bits: x = n ln 2 + r with |r| <= ln 2 / 2 and the exponential series of r up to r^12 / 12! (the next term is
// below 2e-16).  The ranges and signs that the library's function also has to sort out do not occur here.
__device__ __forceinline__ double exp_of_negative(double x) {
    x = fmax(x, -800.0);                     // (zero from -745 on)
    const double n = rint(x * 1.44269504088896340736);
    const double r = fma(n, -1.90821492927058770002e-10, fma(n, -6.93147180369123816490e-01, x));    // ln 2 in two parts, the first of 33 bits
    double p = 1.0 / 479001600.0;
    p = fma(p, r, 1.0 / 39916800.0);
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return ldexp(p, (int)n);
}
// The weight of a logit below or at the row's maximum.  (+inf as the maximum leaves nothing to the others.)
__device__ __forceinline__ double draw_weight(double l, double top, double rate) {
    return l == top ? 1.0 : top == (double)INFINITY ? 0.0 : exp_of_negative((l - top) * rate);
}

// Inclusive sums over the lanes of a wave (and lane 63's, in every lane), with moves between lanes: rows of 16 lanes first, then
// the rows' last lanes into the rows behind them.
template <int kControl, int kRows>
__device__ __forceinline__ uint32_t lane_move(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kControl, kRows, 0xF, false);
}
template <int kControl, int kRows, class T>
__device__ __forceinline__ T lane_move_of(T x) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, lane_move<kControl, kRows>(__builtin_bit_cast(uint32_t, x)));
    } else {
        const unsigned long long v = __builtin_bit_cast(unsigned long long, x);
        const unsigned long long lo = lane_move<kControl, kRows>((uint32_t)v), hi = lane_move<kControl, kRows>((uint32_t)(v >> 32));
        return __builtin_bit_cast(T, hi << 32 | lo);
    }
}
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
    v += lane_move_of<0x111, 0xF>(v);
    v += lane_move_of<0x112, 0xF>(v);
    v += lane_move_of<0x114, 0xF>(v);
    v += lane_move_of<0x118, 0xF>(v);
    v += lane_move_of<0x142, 0xA>(v);
    v += lane_move_of<0x143, 0xC>(v);
    return v;
}
template <class T>
__device__ __forceinline__ T from_lane(T v, int lane) {         // lane: the same in every lane
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else {
        const unsigned long long x = __builtin_bit_cast(unsigned long long, v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane);
        return __builtin_bit_cast(T, (unsigned long long)hi << 32 | lo);
    }
}
template <class T>
__device__ __forceinline__ T wave_sum(T v) { return from_lane(wave_scan(v), 63); }

// A barrier that LDS accesses are ordered by; loads on their way stay so.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Eight consecutive logits, their patterns in 32 bits each.
template <int kBytes>
__device__ __forceinline__ void load_group(const void *row, int g, uint32_t x[8]) {
    if constexpr (kBytes == 2) {
        const uint4 v = stream_load(static_cast<const uint16_t *>(row) + (size_t)g * 8);
        const uint32_t p[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = p[i] & 0xFFFFu; x[2 * i + 1] = p[i] >> 16; }
    } else {
        const uint16_t *at = static_cast<const uint16_t *>(row) + (size_t)g * 16;
        const uint4 v = stream_load(at), w = stream_load(at + 8);
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    }
}
template <int kBytes>
__device__ __forceinline__ uint32_t load_logit(const void *row, int t) {
    if constexpr (kBytes == 2) return static_cast<const uint16_t *>(row)[t];
    else return static_cast<const uint32_t *>(row)[t];
}
// fn(pattern, token) for every allowed token of a row, group of eight by group, groups of a thread kSampleBlock apart.
template <int kBytes, class Fn>
__device__ __forceinline__ void each_allowed(const void *row, const uint8_t *mask, int vocab, int tid, Fn fn) {
    const int whole = vocab >> 3;
    for (int g = tid; g < whole; g += kSampleBlock) {
        const uint32_t mu = mask ? mask[g] : 0xFFu;
        if (mu == 0u) continue;
        uint32_t x[8];
        load_group<kBytes>(row, g, x);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if ((mu >> k) & 1u) fn(x[k], g * 8 + k);
    }
    const int t = whole * 8 + tid;
    if (t < vocab && (!mask || ((mask[t >> 3] >> (t & 7)) & 1u))) fn(load_logit<kBytes>(row, t), t);
}

// The token that is number `rank` (from 0) in ascending id among the allowed ones whose pattern `hit` holds for, by the whole
// block; every thread gets it.  s_part: a word per wave.
template <int kBytes, class Hit>
__device__ int find_token(const void *row, const uint8_t *mask, int vocab, int rank, Hit hit, int *s_part, int *s_found, int tid) {
    const int lane = tid & 63, wave = tid >> 6, whole = vocab >> 3, groups = (vocab + 7) >> 3;
    const unsigned long long lanes_below = (1ull << lane) - 1ull;
    int base = 0;
    if (tid == 0) *s_found = -1;
    __syncthreads();
    for (int g0 = 0; g0 < groups; g0 += kSampleBlock) {
        const int g = g0 + tid;
        uint32_t hits = 0u;
        if (g < groups) {
            const uint32_t mu = (mask ? mask[g] : 0xFFu) & (g < whole ? 0xFFu : (1u << (vocab & 7)) - 1u);
            if (mu != 0u) {
                uint32_t x[8];
                if (g < whole) load_group<kBytes>(row, g, x);
                for (int k = 0; k < 8; ++k)
                    if (((mu >> k) & 1u) && hit(g < whole ? x[k] : load_logit<kBytes>(row, g * 8 + k))) hits |= 1u << k;
            }
        }
        const int mine = __popc(hits);
        int before = 0, sum = 0;
#pragma unroll
        for (int bit = 0; bit < 4; ++bit) {
            const unsigned long long has = __ballot((mine >> bit) & 1);
            before += __popcll(has & lanes_below) << bit;
            sum += __popcll(has) << bit;
        }
        if (lane == 0) s_part[wave] = sum;
        __syncthreads();
        int total = 0;
        before += base;
        for (int w = 0; w < kSampleWaves; ++w) {
            if (w < wave) before += s_part[w];
            total += s_part[w];
        }
        if (rank >= before && rank < before + mine) {
            uint32_t left = hits;
            for (int k = rank - before; k > 0; --k) left &= left - 1u;
            *s_found = g * 8 + __ffs(left) - 1;
        }
        __syncthreads();
        base += total;
        if (base > rank) break;
    }
    return *s_found;
}

__device__ __forceinline__ void put_draw(int b, int token, double logprob, int kept, int32_t *out_tokens, float *out_logprobs, int32_t *out_kept) {
    out_tokens[b] = token;
    if (out_logprobs) out_logprobs[b] = (float)logprob;
    if (out_kept) out_kept[b] = kept;
}

// ------------------------------------------------------------------------------- logits of 16 bits

// A row of 16-bit logits has at most 65,536 different values: how many tokens have each is all that the draw needs, exactly, and
// weights are computed once for a value, in 64 bits.  Counts lie in LDS, 16 bits for a value, the two signs of a magnitude in one word
// (word = pattern without the sign), so that a token is one add without a return and a pattern needs no reordering.
// The order descends through the positive words, then ascends through the negative ones: 1,024 segments of 64 values each.
struct Bf16 {
    static constexpr uint32_t kInf = 0x7F80u;
    __device__ static double value(uint32_t h) { return (double)__uint_as_float(h << 16); }
};
struct F16 {
    static constexpr uint32_t kInf = 0x7C00u;
    __device__ static double value(uint32_t h) { return (double)(float)__builtin_bit_cast(_Float16, (uint16_t)h); }
};
constexpr int kWords = 32768, kSegments = 1024, kHalf = kSegments / 2;
constexpr int kMaxHeavy = 8;                              // segments that can hold 65,536 tokens or more of a row

__device__ __forceinline__ int segment_of(uint32_t word, uint32_t sign) { return sign ? kHalf + (int)(word >> 6) : kHalf - 1 - (int)(word >> 6); }

struct CountTables {
    uint32_t count[kWords];
    double weight[kSegments];                             // summed through the order from the first of every 64 segments on,
    int upto[kSegments];                                  // this segment included
    int heavy_segment[kMaxHeavy];                         // counts that 16 bits do not hold
    uint32_t heavy[kMaxHeavy][64];
    int n_heavy;
};

// Tokens with the value at place `at` (0..63) of a segment.
__device__ __forceinline__ uint32_t word_at(int seg, int at) { return seg < kHalf ? (uint32_t)(kHalf - 1 - seg) * 64u + 63u - at : (uint32_t)(seg - kHalf) * 64u + at; }
__device__ __forceinline__ int count_at(const CountTables &s, int seg, int at) {
    const uint32_t word = word_at(seg, at), both = s.count[word];
    uint32_t c = seg < kHalf ? both & 0xFFFFu : both >> 16;
    for (int i = 0; i < s.n_heavy; ++i) {
        if (s.heavy_segment[i] == seg) return (int)s.heavy[i][at];
        // a positive count beyond 16 bits has carried into the negative one
        if (seg >= kHalf && s.heavy_segment[i] == segment_of(word, 0)) c = (c - (s.heavy[i][63 - at] >> 16)) & 0xFFFFu;
    }
    return (int)c;
}
// A value that the draw may choose: not a NaN, not -inf.
template <class F>
__device__ __forceinline__ bool drawable(int seg, int at) {
    const uint32_t word = word_at(seg, at);
    return word < F::kInf || (word == F::kInf && seg < kHalf);
}
template <class F>
__device__ __forceinline__ double value_at(int seg, int at) { return F::value(word_at(seg, at) | (seg < kHalf ? 0u : 0x8000u)); }

// A place in the order: the value with the token searched for, what lies before the value, and its number of tokens.
struct Place {
    int seg, at, before, count;
    double before_weight, weight;                         // weight: of one of its tokens
};
// Sums through the order over the segments' sixteen parts of 64, in the first sixteen lanes of wave 0 (this part included).
struct Parts { int upto; double weight; };

// The first value whose tokens bring the order to `n` tokens (kByCount), or to more than `border` of weight (kPass), at least
// `border` (kReach); by one wave.  A border that rounding puts behind the last value gives the last one.
enum Search { kByCount, kPass, kReach };
template <class F, Search kHow>
__device__ __forceinline__ Place locate(const CountTables &s, const Parts &parts, int n, double border, double top, double rate, int lane) {
    auto enough = [&](int count, double weight) { return kHow == kByCount ? count >= n : kHow == kPass ? weight > border : weight >= border; };
    // the first of `lanes` lanes whose sums are enough, or the last one's that has a token
    auto first = [&](int lanes, int count, double weight) {
        unsigned long long has = __ballot(lane < lanes && enough(count, weight));
        if (!has) has = __ballot(lane < lanes && count == from_lane(count, lanes - 1));
        return __builtin_amdgcn_readfirstlane(__ffsll(has) - 1);
    };
    const int part = first(16, parts.upto, parts.weight);
    const int upto0 = part ? from_lane(parts.upto, part - 1) : 0;
    const double weight0 = part ? from_lane(parts.weight, part - 1) : 0.0;
    const int upto1 = s.upto[part * 64 + lane] + upto0;
    const double weight1 = s.weight[part * 64 + lane] + weight0;
    const int in_part = first(64, upto1, weight1), seg = part * 64 + in_part;
    const int c = drawable<F>(seg, lane) ? count_at(s, seg, lane) : 0;
    const double w = c ? draw_weight(value_at<F>(seg, lane), top, rate) : 0.0;
    const int upto = wave_scan(c) + (in_part ? from_lane(upto1, in_part - 1) : upto0);
    const double sum = wave_scan(w * c) + (in_part ? from_lane(weight1, in_part - 1) : weight0);
    const unsigned long long has = __ballot(c > 0 && enough(upto, sum));
    const int at = __builtin_amdgcn_readfirstlane(has ? __ffsll(has) - 1 : 63 - __clzll(__ballot(c > 0)));
    Place p;
    p.seg = seg;
    p.at = at;
    p.count = from_lane(c, at);
    p.before = from_lane(upto, at) - p.count;
    p.weight = from_lane(w, at);
    p.before_weight = from_lane(sum - w * c, at);
    return p;
}

// Counts of 16 bits have overflowed: segments are counted in 32 bits and the heavy ones value by value.  A call of its own.
__device__ __noinline__ void count_heavy(CountTables &s, const uint16_t *row, const uint8_t *mask, int vocab) {
    const int tid = threadIdx.x;
    s.upto[tid] = 0;
    __syncthreads();
    each_allowed<2>(row, mask, vocab, tid, [&](uint32_t h, int) { atomicAdd(&s.upto[segment_of(h & 0x7FFFu, h >> 15)], 1); });
    __syncthreads();
    if (tid == 0) {
        int n = 0;
        for (int i = 0; i < kSegments && n < kMaxHeavy; ++i)
            if (s.upto[i] > 0xFFFF) s.heavy_segment[n++] = i;
        s.n_heavy = n;
    }
    __syncthreads();
    const int n_heavy = s.n_heavy;
    for (int i = tid; i < n_heavy * 64; i += kSampleBlock) s.heavy[i / 64][i % 64] = 0u;
    s.upto[tid] = 0;
    __syncthreads();
    each_allowed<2>(row, mask, vocab, tid, [&](uint32_t h, int) {
        const int seg = segment_of(h & 0x7FFFu, h >> 15);
        for (int i = 0; i < n_heavy; ++i)
            if (s.heavy_segment[i] == seg) atomicAdd(&s.heavy[i][seg < kHalf ? 63 - (h & 63u) : h & 63u], 1u);
    });
    __syncthreads();
}

// What wave 0 has drawn: the pattern (0 stands for both zeros), the token's rank among its equals by id,
// its weight, and the tokens kept with their weight.
struct Drawn { uint32_t word, sign; int rank, kept; double weight, total; };

// By wave 0, behind the summed segments: what is kept, and the draw.
template <class F>
__device__ __forceinline__ Drawn draw_from_counts(const CountTables &s, const Parts &parts, const RowDraw &draw, double top, int likely, int lane) {
    const int n_all = from_lane(parts.upto, 15);
    int n = n_all;
    double total = from_lane(parts.weight, 15);
    auto first_tokens = [&](int count) {                   // their weight
        const Place p = locate<F, kByCount>(s, parts, count, 0.0, top, draw.rate, lane);
        return p.before_weight + p.weight * (count - p.before);
    };
    if (draw.top_k > 0 && draw.top_k < n) { n = draw.top_k; total = first_tokens(n); }
    int kept = n;
    if (draw.top_p < 1.0) {
        const double border = draw.top_p * total;
        const Place p = locate<F, kReach>(s, parts, 0, border, top, draw.rate, lane);
        const double r = ceil((border - p.before_weight) / p.weight);              // tokens of the value with less than the border before them
        kept = min(kept, p.before + (r >= p.count ? p.count : r >= 1.0 ? (int)r : 1));
    }
    if (draw.min_p > 0.0) kept = min(kept, likely);
    kept = max(kept, 1);
    if (kept < n) total = first_tokens(kept);
    const double border = draw.uniform * total;
    Place p = locate<F, kPass>(s, parts, 0, border, top, draw.rate, lane);
    const double r = floor((border - p.before_weight) / p.weight);
    Drawn d;
    d.rank = r >= p.count ? p.count - 1 : r >= 1.0 ? (int)r : 0;
    if (p.before + d.rank >= kept) {                       // (rounding, or a number that is not below 1: the last of those kept)
        p = locate<F, kByCount>(s, parts, kept, 0.0, top, draw.rate, lane);
        d.rank = kept - 1 - p.before;
    }
    d.word = word_at(p.seg, p.at);
    d.sign = p.seg < kHalf ? 0u : 0x8000u;
    if (d.word == 0u) {                                    // -0 and +0 are one value
        if (d.sign) d.rank += count_at(s, kHalf - 1, 63);
        d.sign = 0u;
    }
    d.kept = kept;
    d.weight = p.weight;
    d.total = total;
    return d;
}

// Two tokens of 16 bits in a register: which halves of x are equal to those of `pair` where `care` has bits, as zero halves.
__device__ __forceinline__ uint32_t differing(uint32_t x, uint32_t pair, uint32_t care) { return (x ^ pair) & care; }
typedef unsigned short PackedU16 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t packed_min(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(PackedU16, a), __builtin_bit_cast(PackedU16, b)));
}
__device__ __forceinline__ uint32_t packed_signs(uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(PackedU16, x) >> 15); }

// One block a row.  A wave's groups of eight tokens are neighbours, kG rounds of 64; a row of more than a block's kG * 8,192 tokens
// (kMany) goes through in chunks and is read again for the token's id.
template <class F, int kG, bool kMany>
__global__ __launch_bounds__(kSampleBlock) void sample_counts_kernel(const uint16_t *__restrict__ logits, const uint32_t *__restrict__ bitmask,
                                                                    int vocab, int64_t row_stride, int n_words, SampleRows rows,
                                                                    int32_t *__restrict__ out_tokens, float *__restrict__ out_logprobs,
                                                                    int32_t *__restrict__ out_kept) {
    constexpr int kAhead = kG < 8 ? kG : 8, kLook = kWords / 256 / kSampleWaves;           // groups in flight; looks at 256 words a wave
    __shared__ __align__(16) CountTables s;
    __shared__ uint2 s_ones[16];                          // four mask bits -> 1 or 0 in the halves of two registers
    __shared__ uint16_t s_busy[kSegments];                // segments that have tokens
    __shared__ int s_first, s_likely, s_seen, s_n_busy, s_part[kSampleWaves];
    __shared__ Drawn s_drawn;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
    const uint16_t *row = logits + (size_t)b * row_stride;
    const uint8_t *mask = bitmask ? reinterpret_cast<const uint8_t *>(bitmask + (size_t)b * n_words) : nullptr;
    const int whole = vocab >> 3, rest = vocab & 7, chunks = kMany ? (whole + kG * kSampleBlock - 1) / (kG * kSampleBlock) : 1;
    uint4 v[kG], v_rest;                                   // v_rest: the last group, not whole, of the last wave's first lane
    uint32_t packed[(kG + 3) / 4], m_rest = 0u;            // mask bytes of the groups, 0 behind the row
    auto group_of = [&](int chunk, int u) { return (chunk * kSampleWaves + wave) * (kG * 64) + u * 64 + lane; };
    auto load_masks = [&](int chunk) {
        uint32_t m[kG];
#pragma unroll
        for (int u = 0; u < kG; ++u) m[u] = mask ? mask[min(group_of(chunk, u), max(whole - 1, 0))] : 0xFFu;
#pragma unroll
        for (int u = 0; u < kG; ++u) packed[u / 4] = (u & 3 ? packed[u / 4] : 0u) | (group_of(chunk, u) < whole ? m[u] : 0u) << (8 * (u & 3));
    };
    auto load = [&](int chunk, int u) { v[u] = stream_load_at(row, (uint32_t)min(group_of(chunk, u), whole - 1) * 16u); };
    auto load_all = [&](int chunk, int from, int to) {
        if (kG > 1 || whole > 0) {                         // (no branch around the loads of the longer rows)
#pragma unroll
            for (int u = from; u < to; ++u) load(chunk, u);
        }
    };
    uint32_t seen = 0u;
    auto count_group = [&](uint4 group, uint32_t a) {
        if (a == 0u) return;
        seen += __popc(a);
        const uint2 first = s_ones[a & 15u], second = s_ones[a >> 4];
        const uint32_t x[4] = {group.x, group.y, group.z, group.w}, one[4] = {first.x, first.y, second.x, second.y};
        char *table = reinterpret_cast<char *>(s.count);
#pragma unroll
        for (int i = 0; i < 4; ++i) {                      // (a masked token adds nothing, to its own word)
            const uint32_t word = x[i] & 0x7FFF7FFFu, negative = one[i] & packed_signs(x[i]), positive = one[i] ^ negative;
            atomicAdd(reinterpret_cast<uint32_t *>(table + ((word & 0xFFFFu) << 2)), __builtin_amdgcn_perm(negative, positive, 0x05040100u));
            atomicAdd(reinterpret_cast<uint32_t *>(table + ((word >> 16) << 2)), __builtin_amdgcn_perm(negative, positive, 0x07060302u));
        }
    };
    // (1) counts
    load_masks(0);
    load_all(0, 0, kAhead);
    if (rest && wave == kSampleWaves - 1 && lane == 0) {
        uint32_t x[4] = {0u, 0u, 0u, 0u};
        for (int k = 0; k < rest; ++k) x[k >> 1] |= (uint32_t)row[whole * 8 + k] << (16 * (k & 1));
        v_rest = make_uint4(x[0], x[1], x[2], x[3]);
        m_rest = (mask ? mask[whole] : 0xFFu) & ((1u << rest) - 1u);
    }
    const RowDraw draw = row_draw(rows, b);
    for (int i = tid; i < kWords / 4; i += kSampleBlock) reinterpret_cast<uint4 *>(s.count)[i] = make_uint4(0u, 0u, 0u, 0u);
    s.upto[tid] = 0;
    s.weight[tid] = 0.0;
    if (tid < 16) s_ones[tid] = make_uint2((tid & 1) | (tid & 2) << 15, (tid >> 2 & 1) | (tid >> 2 & 2) << 15);
    if (tid == 0) { s.n_heavy = 0; s_first = kSegments; s_likely = 0; s_seen = 0; s_n_busy = 0; }
    lds_barrier();
    for (int chunk = 0; chunk < chunks; ++chunk) {
        if (kMany && chunk > 0) {
            load_masks(chunk);
            load_all(chunk, 0, kAhead);
        }
#pragma unroll
        for (int u = 0; u < kG; ++u) {
            if (u + kAhead < kG) load_all(chunk, u + kAhead, u + kAhead + 1);
            __builtin_amdgcn_sched_barrier(0);
            count_group(v[u], (packed[u / 4] >> (8 * (u & 3))) & 0xFFu);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    count_group(v_rest, m_rest);
    lds_barrier();
    // (2) the segments with tokens, the first of them, and whether the counts are whole
    int first = kSegments;
    auto add_busy = [&](int seg) {                         // by one lane
        s_busy[atomicAdd(&s_n_busy, 1)] = (uint16_t)seg;
    };
    uint32_t counted = 0u;
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
        const uint32_t word = (uint32_t)(wave + i * kSampleWaves) * 256u + (uint32_t)lane * 4u;
        const uint4 c = *reinterpret_cast<const uint4 *>(s.count + word);
        counted = __builtin_amdgcn_sad_u16(c.x, 0u, __builtin_amdgcn_sad_u16(c.y, 0u, __builtin_amdgcn_sad_u16(c.z, 0u, __builtin_amdgcn_sad_u16(c.w, 0u, counted))));
        uint32_t any = c.x | c.y | c.z | c.w;
        if (word >= F::kInf) any = word == F::kInf ? c.x & 0xFFFFu : 0u;   // +inf, no -inf, no NaNs
        const unsigned long long positive = __ballot((any & 0xFFFFu) != 0u), negative = __ballot(any > 0xFFFFu);
        if ((positive | negative) == 0ull) continue;
        // lane 0..3: the positive segment of these 64 words, 4..7 the negative one
        const uint32_t sixteen = (uint32_t)((lane & 4 ? negative : positive) >> (16 * (lane & 3))) & 0xFFFFu;
        if (lane < 8 && sixteen != 0u) {
            const int seg = segment_of((uint32_t)(wave + i * kSampleWaves) * 256u + (uint32_t)(lane & 3) * 64u, lane & 4);
            first = min(first, seg);
            add_busy(seg);
        }
    }
    if (first < kSegments) atomicMin(&s_first, first);
    if (vocab > 0xFFFF) {
        // Counts beyond 16 bits carry or vanish, and the sum tells.
        const int missing = wave_sum((int)(seen - counted));
        if (lane == 0 && missing != 0) atomicAdd(&s_seen, missing);
    }
    lds_barrier();
    if (s_seen != 0) {
        count_heavy(s, row, mask, vocab);
        if (tid == 0) { s_n_busy = 0; s_first = kSegments; }
        lds_barrier();
        for (int j = wave; j < kSegments; j += kSampleWaves)
            if (__any(drawable<F>(j, lane) && count_at(s, j, lane) > 0) && lane == 0) { add_busy(j); atomicMin(&s_first, j); }
        lds_barrier();
    }
    first = s_first;
    if (first == kSegments) {
        // nothing to draw from: the first token of -inf, as for the arg max, or none
        const int token = find_token<2>(row, mask, vocab, 0, [=](uint32_t h) { return h == (F::kInf | 0x8000u); }, s_part, &s_seen, tid);
        if (tid == 0) put_draw(b, token, token < 0 ? -(double)INFINITY : 0.0, token < 0 ? 0 : 1, out_tokens, out_logprobs, out_kept);
        return;
    }
    // (3) every segment's count and weight
    const double top = value_at<F>(first, __ffsll(__ballot(drawable<F>(first, lane) && count_at(s, first, lane) > 0)) - 1);
    const int n_busy = s_n_busy;
    int likely = 0;
    for (int i = wave; i < n_busy; i += kSampleWaves) {
        const int seg = __builtin_amdgcn_readfirstlane(s_busy[i]);
        const int c = drawable<F>(seg, lane) ? count_at(s, seg, lane) : 0;
        const double w = c ? draw_weight(value_at<F>(seg, lane), top, draw.rate) : 0.0;
        if (w >= draw.min_p) likely += c;
        const int n = wave_scan(c);
        const double sum = wave_scan(w * c);
        if (lane == 63) { s.upto[seg] = n; s.weight[seg] = sum; }
    }
    if (draw.min_p > 0.0) {
        likely = wave_sum(likely);
        if (lane == 0) atomicAdd(&s_likely, likely);
    }
    lds_barrier();
    // (4) sums through the order, a part of 64 segments a wave; the draw by wave 0
    s.upto[tid] = wave_scan(s.upto[tid]);
    s.weight[tid] = wave_scan(s.weight[tid]);
    lds_barrier();
    if (wave == 0) {
        Parts parts;
        parts.upto = wave_scan(s.upto[(lane & 15) * 64 + 63]);
        parts.weight = wave_scan(s.weight[(lane & 15) * 64 + 63]);                         // (the first sixteen lanes' are theirs)
        const Drawn d = draw_from_counts<F>(s, parts, draw, top, s_likely, lane);
        if (lane == 0) s_drawn = d;
    }
    lds_barrier();
    // (5) the token's id: number `rank` among the allowed tokens with the pattern, by ascending id
    const uint32_t word = s_drawn.word, pattern = word | s_drawn.sign, care = word ? 0xFFFFFFFFu : 0x7FFF7FFFu, pair = pattern | pattern << 16;
    const int rank = s_drawn.rank;
    auto hits_of = [&](uint4 group, uint32_t a) {          // bit k: token k of the group
        const uint32_t x[4] = {group.x, group.y, group.z, group.w};
        uint32_t hits = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t y = differing(x[i], pair, care);
            hits |= ((y & 0xFFFFu) == 0u ? 1u << (2 * i) : 0u) | (y < 0x10000u ? 2u << (2 * i) : 0u);
        }
        return hits & a;
    };
    int base = 0;
    for (int chunk = 0; chunk < chunks; ++chunk) {
        if (kMany) {
            load_masks(chunk);
            load_all(chunk, 0, kG);
        }
        // a thread with an equal among its tokens, masked or not, looks closer
        uint32_t least = 0xFFFFFFFFu;
#pragma unroll
        for (int u = 0; u < kG; ++u) {
            least = packed_min(least, packed_min(packed_min(differing(v[u].x, pair, care), differing(v[u].y, pair, care)),
                                                 packed_min(differing(v[u].z, pair, care), differing(v[u].w, pair, care))));
        }
        int mine = 0;
        uint32_t with_hits = 0u;                           // rounds
        if ((least & 0xFFFFu) == 0u || least < 0x10000u) {
#pragma unroll
            for (int u = 0; u < kG; ++u) {
                const int n = __popc(hits_of(v[u], packed[u / 4] >> (8 * (u & 3)) & 0xFFu));
                mine += n;
                with_hits |= (n ? 1u : 0u) << u;
            }
        }
        const uint32_t hits_rest = chunk == chunks - 1 ? hits_of(v_rest, m_rest) : 0u;     // (m_rest is 0 but in one lane)
        mine += __popc(hits_rest);
        const int sum = __any(mine != 0) ? wave_sum(mine) : 0;
        if (lane == 0) s_part[wave] = sum;
        lds_barrier();
        const int upto = wave_scan(lane < kSampleWaves ? s_part[lane] : 0), total = from_lane(upto, kSampleWaves - 1);
        int before = base + (wave ? from_lane(upto, wave - 1) : 0);
        if (rank >= before && rank < before + sum) {       // the wave that has it: round by round
            auto round = [&](uint32_t hits, int g) {
                const int n = __popc(hits), through = wave_scan(n), place = before + through - n;
                if (rank >= place && rank < place + n) {
                    uint32_t left = hits;
                    for (int k = rank - place; k > 0; --k) left &= left - 1u;
                    out_tokens[b] = g * 8 + __ffs(left) - 1;
                }
                before += from_lane(through, 63);
            };
#pragma unroll
            for (int u = 0; u < kG; ++u)
                if (__any((with_hits >> u) & 1u)) round(hits_of(v[u], packed[u / 4] >> (8 * (u & 3)) & 0xFFu), group_of(chunk, u));
            round(hits_rest, whole);
        }
        base += total;
        if (!kMany || base > rank) break;
        lds_barrier();
    }
    if (tid == 0) {
        if (out_logprobs) out_logprobs[b] = (float)log(s_drawn.weight / s_drawn.total);
        if (out_kept) out_kept[b] = s_drawn.kept;
    }
}

template <class F>
void launch_counts(const uint16_t *logits, const uint32_t *bitmask, int batch, int vocab, int64_t row_stride, int n_words, const SampleRows &rows,
                   int32_t *out_tokens, float *out_logprobs, int32_t *out_kept, hipStream_t stream) {
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(batch), dim3(kSampleBlock), 0, stream, logits, bitmask, vocab, row_stride, n_words, rows, out_tokens,
                           out_logprobs, out_kept);
    };
    const int rounds = (vocab + kSampleBlock * 8 - 1) / (kSampleBlock * 8);
    if (rounds <= 1) go(sample_counts_kernel<F, 1, false>);
    else if (rounds <= 4) go(sample_counts_kernel<F, 4, false>);
    else if (rounds <= 8) go(sample_counts_kernel<F, 8, false>);
    else if (rounds <= 12) go(sample_counts_kernel<F, 12, false>);
    else if (rounds <= 16) go(sample_counts_kernel<F, 16, false>);
    else if (rounds <= 20) go(sample_counts_kernel<F, 20, false>);
    else go(sample_counts_kernel<F, 8, true>);
}

// ------------------------------------------------------------------------------- logits of 32 bits

// Logits of 32 bits have too many values to count.  A token is put into one of 4,096 classes (the first 12 bits of a key whose order is
// that of the draw), tokens and weights of every class are summed, and a place is found by its class first; then the tokens of that class are
// looked at once more, by the next ten bits of their keys and by the last ten.  Weights are summed as whole numbers, in units so small that the
// vocabulary's sum just fits 64 bits (2^-45 for 128,256 tokens): in whatever order the tokens arrive, the sums are the same.
constexpr int kClasses = 4096, kDigits = 1024, kListed = 8192;

__device__ __forceinline__ uint32_t falling_key(uint32_t bits) {            // ascending keys: descending numbers; -0 as +0
    if (bits == 0x80000000u) bits = 0u;
    return (bits & 0x80000000u) ? bits : ~(bits | 0x80000000u);
}
__device__ __forceinline__ float of_falling_key(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key : ~key & 0x7FFFFFFFu); }
constexpr uint32_t kKeyPosInf = 0x007FFFFFu, kKeyNegInf = 0xFF800000u;      // NaNs lie outside

struct ClassTables {
    unsigned long long weight[kClasses];      // through the order, the class included
    int upto[kClasses];
    unsigned long long digit_weight[kDigits];
    int digit_count[kDigits];
    uint32_t listed_key[kListed];
    int listed_id[kListed];
    unsigned long long part[kSampleWaves];
    int part_count[kSampleWaves];
    uint32_t best;
    int neg_inf, likely, listed, at, found;
    int before;
    unsigned long long before_weight;
};

__global__ __launch_bounds__(kSampleBlock) void sample_classes_kernel(const uint32_t *__restrict__ logits, const uint32_t *__restrict__ bitmask,
                                                                     int vocab, int64_t row_stride, int n_words, int unit_bits, SampleRows rows,
                                                                     int32_t *__restrict__ out_tokens, float *__restrict__ out_logprobs,
                                                                     int32_t *__restrict__ out_kept) {
    __shared__ ClassTables s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
    const uint32_t *row = logits + (size_t)b * row_stride;
    const uint8_t *mask = bitmask ? reinterpret_cast<const uint8_t *>(bitmask + (size_t)b * n_words) : nullptr;
    const RowDraw draw = row_draw(rows, b);
    const double unit = ldexp(1.0, unit_bits);
    if (tid == 0) { s.best = kKeyNegInf; s.neg_inf = 0; s.likely = 0; }
    for (int i = tid; i < kClasses; i += kSampleBlock) { s.weight[i] = 0ull; s.upto[i] = 0; }
    __syncthreads();
    uint32_t best = kKeyNegInf;
    each_allowed<4>(row, mask, vocab, tid, [&](uint32_t x, int) {
        const uint32_t key = falling_key(x);
        if (key >= kKeyPosInf) best = min(best, key);
    });
    for (int step = 32; step > 0; step /= 2) best = min(best, (uint32_t)__shfl_xor((int)best, step));
    if (lane == 0) atomicMin(&s.best, best);
    __syncthreads();
    best = s.best;
    if (best >= kKeyNegInf) {                  // nothing to draw from
        const int token = find_token<4>(row, mask, vocab, 0, [](uint32_t x) { return x == 0xFF800000u; }, s.part_count, &s.found, tid);
        if (tid == 0) put_draw(b, token, token < 0 ? -(double)INFINITY : 0.0, token < 0 ? 0 : 1, out_tokens, out_logprobs, out_kept);
        return;
    }
    const double top = (double)of_falling_key(best);
    auto candidate = [&](uint32_t key) { return key >= kKeyPosInf && key < kKeyNegInf; };
    auto weight_of = [&](uint32_t key) { return draw_weight((double)of_falling_key(key), top, draw.rate); };
    auto in_units = [&](double w) { return (unsigned long long)(w * unit + 0.5); };
    int likely = 0;
    each_allowed<4>(row, mask, vocab, tid, [&](uint32_t x, int) {
        const uint32_t key = falling_key(x);
        if (!candidate(key)) return;
        const double w = weight_of(key);
        if (w >= draw.min_p) ++likely;
        atomicAdd(&s.upto[key >> 20], 1);
        atomicAdd(&s.weight[key >> 20], in_units(w));
    });
    likely = wave_sum(likely);
    if (lane == 0) atomicAdd(&s.likely, likely);
    __syncthreads();
    // sums through the order, in place; kPer entries a thread
    auto scan = [&](int *count, unsigned long long *weight, auto per) {
        constexpr int kPer = decltype(per)::value;
        int c[kPer];
        unsigned long long w[kPer];
        for (int i = 0; i < kPer; ++i) {
            c[i] = count[tid * kPer + i] + (i ? c[i - 1] : 0);
            w[i] = weight[tid * kPer + i] + (i ? w[i - 1] : 0ull);
        }
        const int cs = wave_scan(c[kPer - 1]);
        const unsigned long long ws = wave_scan(w[kPer - 1]);
        if (lane == 63) { s.part_count[wave] = cs; s.part[wave] = ws; }
        __syncthreads();
        int c0 = cs - c[kPer - 1];
        unsigned long long w0 = ws - w[kPer - 1];
        for (int v = 0; v < wave; ++v) { c0 += s.part_count[v]; w0 += s.part[v]; }
        for (int i = 0; i < kPer; ++i) { count[tid * kPer + i] = c[i] + c0; weight[tid * kPer + i] = w[i] + w0; }
        __syncthreads();
    };
    scan(s.upto, s.weight, std::integral_constant<int, kClasses / kSampleBlock>());
    const int n_all = s.upto[kClasses - 1];

    struct At { uint32_t key; int before, count; unsigned long long before_weight; };
    int listed_class = -1;
    bool complete = false;                     // the class's tokens are all in the list
    // the first key whose tokens bring the order to `n` tokens (how 0), to more than `border` (1), to at least `border` (2); by the block
    auto locate = [&](int how, int n, double border) -> At {
        auto enough = [&](int count, unsigned long long weight) { return how == 0 ? count >= n : how == 1 ? (double)weight > border : (double)weight >= border; };
        // the first of `entries` sums that is enough; the last one that has a token where rounding leaves none
        auto choose = [&](const int *count, const unsigned long long *weight, int entries, int c0, unsigned long long w0) {
            const int last = count[entries - 1];
            if (tid == 0) s.at = entries;
            __syncthreads();
            for (int i = tid; i < entries; i += kSampleBlock) {
                const int before = i ? count[i - 1] : 0;
                if (count[i] > before && (enough(c0 + count[i], w0 + weight[i]) || count[i] == last)) atomicMin(&s.at, i);
            }
            __syncthreads();
            const int at = s.at;
            __syncthreads();
            return at;
        };
        const int cls = choose(s.upto, s.weight, kClasses, 0, 0ull);
        At a;
        a.before = cls ? s.upto[cls - 1] : 0;
        a.before_weight = cls ? s.weight[cls - 1] : 0ull;
        if (cls != listed_class) {
            listed_class = cls;
            complete = s.upto[cls] - a.before <= kListed;
            if (tid == 0) s.listed = 0;
            __syncthreads();
            if (complete)
                each_allowed<4>(row, mask, vocab, tid, [&](uint32_t x, int t) {
                    const uint32_t key = falling_key(x);
                    if (!candidate(key) || (int)(key >> 20) != cls) return;
                    const int i = atomicAdd(&s.listed, 1);
                    s.listed_key[i] = key;
                    s.listed_id[i] = t;
                });
            __syncthreads();
        }
        uint32_t prefix = (uint32_t)cls;
        for (int level = 0; level < 2; ++level) {
            const int shift = level ? 0 : 10;
            s.digit_count[tid] = 0;
            s.digit_weight[tid] = 0ull;
            __syncthreads();
            auto add = [&](uint32_t key) {
                if (!candidate(key) || key >> (shift + 10) != prefix) return;
                atomicAdd(&s.digit_count[(key >> shift) & 1023u], 1);
                atomicAdd(&s.digit_weight[(key >> shift) & 1023u], in_units(weight_of(key)));
            };
            if (complete) for (int i = tid; i < s.listed; i += kSampleBlock) add(s.listed_key[i]);
            else each_allowed<4>(row, mask, vocab, tid, [&](uint32_t x, int) { add(falling_key(x)); });
            __syncthreads();
            scan(s.digit_count, s.digit_weight, std::integral_constant<int, 1>());
            const int digit = choose(s.digit_count, s.digit_weight, kDigits, a.before, a.before_weight);
            const int c = digit ? s.digit_count[digit - 1] : 0;
            a.count = s.digit_count[digit] - c;
            a.before += c;
            a.before_weight += digit ? s.digit_weight[digit - 1] : 0ull;
            prefix = prefix << 10 | (uint32_t)digit;
            __syncthreads();
        }
        a.key = prefix;
        return a;
    };
    int n = n_all;
    double total = (double)s.weight[kClasses - 1];
    auto first_tokens = [&](int count) {
        const At a = locate(0, count, 0.0);
        return (double)(a.before_weight + in_units(weight_of(a.key)) * (unsigned long long)(count - a.before));
    };
    if (draw.top_k > 0 && draw.top_k < n) { n = draw.top_k; total = first_tokens(n); }
    int kept = n;
    if (draw.top_p < 1.0) {
        const double border = draw.top_p * total;
        const At a = locate(2, 0, border);
        const double r = ceil((border - (double)a.before_weight) / (double)in_units(weight_of(a.key)));
        kept = min(kept, a.before + (r >= a.count ? a.count : r >= 1.0 ? (int)r : 1));
    }
    if (draw.min_p > 0.0) kept = min(kept, s.likely);
    kept = max(kept, 1);
    if (kept < n) total = first_tokens(kept);
    const double border = draw.uniform * total;
    At a = locate(1, 0, border);
    const double r = floor((border - (double)a.before_weight) / (double)in_units(weight_of(a.key)));
    int rank = r >= a.count ? a.count - 1 : r >= 1.0 ? (int)r : 0;
    if (a.before + rank >= kept) {
        a = locate(0, kept, 0.0);
        rank = kept - 1 - a.before;
    }
    int token;
    if (complete && a.count == 1) {
        for (int i = tid; i < s.listed; i += kSampleBlock)
            if (s.listed_key[i] == a.key) s.found = s.listed_id[i];
        __syncthreads();
        token = s.found;
    } else {
        const uint32_t key = a.key;
        token = find_token<4>(row, mask, vocab, rank, [=](uint32_t x) { return falling_key(x) == key; }, s.part_count, &s.found, tid);
    }
    if (tid == 0) put_draw(b, token, log(weight_of(a.key) * unit / total), kept, out_tokens, out_logprobs, out_kept);
}

}  // namespace

hipError_t launch_masked_sample(const void *logits, LogitType type, const uint32_t *bitmask, int batch, int vocab, int64_t row_stride,
                                const SampleRows &rows, int32_t *out_tokens, float *out_logprobs, int32_t *out_kept, hipStream_t stream) {
    if (batch == 0) return hipSuccess;
    const int n_words = (vocab + 31) / 32;
    if (type == kLogitBf16)
        launch_counts<Bf16>(static_cast<const uint16_t *>(logits), bitmask, batch, vocab, row_stride, n_words, rows, out_tokens, out_logprobs, out_kept, stream);
    else if (type == kLogitF16)
        launch_counts<F16>(static_cast<const uint16_t *>(logits), bitmask, batch, vocab, row_stride, n_words, rows, out_tokens, out_logprobs, out_kept, stream);
    else {
        int bits = 62;                          // the vocabulary's sum of weights stays below 2^63
        while (bits > 30 && ((int64_t)1 << (62 - bits)) < vocab) --bits;
        hipLaunchKernelGGL(sample_classes_kernel, dim3(batch), dim3(kSampleBlock), 0, stream, static_cast<const uint32_t *>(logits), bitmask, vocab, row_stride,
                           n_words, bits, rows, out_tokens, out_logprobs, out_kept);
    }
    return hipGetLastError();
}

}  // namespace pre3
