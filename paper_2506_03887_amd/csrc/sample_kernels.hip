// gfx950 kernels of the sampler behind the mask: one token a row by temperature, top-k, top-p and min-p, from one given random
// number a row.  The logits are read, nothing is written back.
//
// The order of the draw is that of the logits, descending, equal ones by ascending id; w = exp((l - max) / temperature).  Top-k,
// top-p and min-p each keep a prefix of that order, so what is drawn from is its first n tokens, and everything that has to be found
// is a place in the order: the token number n, or the token at which the summed weights pass a border.
#include <hip/hip_runtime.h>

#include <cstdint>

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
// The weight of a logit below or at the row's maximum.  (+inf as the maximum leaves nothing to the others.)
__device__ __forceinline__ double draw_weight(double l, double top, double rate) {
    return l == top ? 1.0 : top == (double)INFINITY ? 0.0 : exp((l - top) * rate);
}

__device__ __forceinline__ double wave_scan(double v, int lane) {       // inclusive
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
        const double o = __shfl_up(v, step);
        if (lane >= step) v += o;
    }
    return v;
}
template <class T>
__device__ __forceinline__ T wave_scan_int(T v, int lane) {
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
        const T o = __shfl_up(v, step);
        if (lane >= step) v += o;
    }
    return v;
}
template <class T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
    for (int step = 32; step > 0; step /= 2) v += __shfl_xor(v, step);
    return v;
}

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
    double weight[kSegments];                             // summed through the order, this segment included
    int upto[kSegments];
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
// The first value whose tokens bring the order to `n` tokens (kByCount), or to more than `border` of weight (at least `border`:
// kReach); by one wave.  A border that rounding puts behind the last value gives the last one.
enum Search { kByCount, kPass, kReach };
template <class F, Search kHow>
__device__ __forceinline__ Place locate(const CountTables &s, int n, double border, double top, double rate, int n_all, int lane) {
    auto enough = [&](int count, double weight) { return kHow == kByCount ? count >= n : kHow == kPass ? weight > border : weight >= border; };
    unsigned long long has = __ballot(enough(s.upto[lane * 16 + 15], s.weight[lane * 16 + 15]));
    int seg = has ? (__ffsll(has) - 1) * 16 : 0;
    if (has) {
        has = __ballot(lane < 16 && enough(s.upto[seg + (lane & 15)], s.weight[seg + (lane & 15)]));
        seg += __ffsll(has) - 1;
    } else {                                              // the segment of the last token
        for (int i = 0; i < 16; ++i) {
            has = __ballot(s.upto[i * 64 + lane] >= n_all);
            if (has) { seg = i * 64 + __ffsll(has) - 1; break; }
        }
    }
    const int c = drawable<F>(seg, lane) ? count_at(s, seg, lane) : 0;
    const double w = c ? draw_weight(value_at<F>(seg, lane), top, rate) : 0.0;
    const int upto = wave_scan_int(c, lane) + (seg ? s.upto[seg - 1] : 0);
    const double sum = wave_scan(w * c, lane) + (seg ? s.weight[seg - 1] : 0.0);
    has = __ballot(c > 0 && enough(upto, sum));
    if (!has) has = 1ull << (63 - __clzll(__ballot(c > 0)));
    const int at = __ffsll(has) - 1;
    Place p;
    p.seg = seg;
    p.at = at;
    p.count = __shfl(c, at);
    p.before = __shfl(upto, at) - p.count;
    p.weight = __shfl(w, at);
    p.before_weight = __shfl(sum - w * c, at);
    return p;
}

template <class F>
__global__ __launch_bounds__(kSampleBlock) void sample_counts_kernel(const uint16_t *__restrict__ logits, const uint32_t *__restrict__ bitmask,
                                                                    int vocab, int64_t row_stride, int n_words, SampleRows rows,
                                                                    int32_t *__restrict__ out_tokens, float *__restrict__ out_logprobs,
                                                                    int32_t *__restrict__ out_kept) {
    __shared__ CountTables s;
    __shared__ double s_part[kSampleWaves];
    __shared__ int s_part_count[kSampleWaves], s_first, s_likely, s_seen, s_counted, s_rank, s_found;
    __shared__ uint32_t s_word, s_sign;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
    const uint16_t *row = logits + (size_t)b * row_stride;
    const uint8_t *mask = bitmask ? reinterpret_cast<const uint8_t *>(bitmask + (size_t)b * n_words) : nullptr;
    const RowDraw draw = row_draw(rows, b);
    for (int i = tid; i < kWords; i += kSampleBlock) s.count[i] = 0u;
    if (tid == 0) { s.n_heavy = 0; s_first = kSegments; s_likely = 0; s_seen = 0; s_counted = 0; }
    __syncthreads();
    int seen = 0;
    each_allowed<2>(row, mask, vocab, tid, [&](uint32_t h, int) {
        atomicAdd(&s.count[h & 0x7FFFu], (h & 0x8000u) ? 0x10000u : 1u);
        ++seen;
    });
    __syncthreads();
    if (vocab > 0xFFFF) {
        // Counts beyond 16 bits carry or vanish, and the sum tells.  Rows of so many equal logits are counted by segments, the
        // heavy ones value by value.
        int counted = 0;
        for (int i = tid; i < kWords; i += kSampleBlock) counted += (int)((s.count[i] & 0xFFFFu) + (s.count[i] >> 16));
        seen = wave_sum(seen);
        counted = wave_sum(counted);
        if (lane == 0) { atomicAdd(&s_seen, seen); atomicAdd(&s_counted, counted); }
        __syncthreads();
        if (s_seen != s_counted) {
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
            __syncthreads();
            each_allowed<2>(row, mask, vocab, tid, [&](uint32_t h, int) {
                const int seg = segment_of(h & 0x7FFFu, h >> 15);
                for (int i = 0; i < n_heavy; ++i)
                    if (s.heavy_segment[i] == seg) atomicAdd(&s.heavy[i][seg < kHalf ? 63 - (h & 63u) : h & 63u], 1u);
            });
            __syncthreads();
        }
    }
    // the first segment with a token, and its best value
    for (int j = wave; j < kSegments; j += kSampleWaves) {
        if (__any(drawable<F>(j, lane) && count_at(s, j, lane) > 0)) {
            if (lane == 0) atomicMin(&s_first, j);
            break;
        }
    }
    __syncthreads();
    const int first = s_first;
    if (first < kSegments) {
        const int best_at = __ffsll(__ballot(drawable<F>(first, lane) && count_at(s, first, lane) > 0)) - 1;
        const double top = value_at<F>(first, best_at);
        // every segment's count and weight, then summed through the order
        int likely = 0;
        for (int j = wave; j < kSegments; j += kSampleWaves) {
            const int c = drawable<F>(j, lane) ? count_at(s, j, lane) : 0;
            int n = 0;
            double sum = 0.0;
            if (__any(c > 0)) {
                const double w = c ? draw_weight(value_at<F>(j, lane), top, draw.rate) : 0.0;
                if (w >= draw.min_p) likely += c;
                n = wave_sum(c);
                sum = wave_sum(w * c);
            }
            if (lane == 0) { s.upto[j] = n; s.weight[j] = sum; }
        }
        likely = wave_sum(likely);
        if (lane == 0) atomicAdd(&s_likely, likely);
        __syncthreads();
        int upto = wave_scan_int(s.upto[tid], lane);
        double sum = wave_scan(s.weight[tid], lane);
        if (lane == 63) { s_part_count[wave] = upto; s_part[wave] = sum; }
        __syncthreads();
        for (int w = 0; w < wave; ++w) { upto += s_part_count[w]; sum += s_part[w]; }
        s.upto[tid] = upto;
        s.weight[tid] = sum;
        __syncthreads();
        if (wave == 0) {
            const int n_all = s.upto[kSegments - 1];
            int n = n_all;
            double total = s.weight[kSegments - 1];
            auto first_tokens = [&](int count) {           // their weight
                const Place p = locate<F, kByCount>(s, count, 0.0, top, draw.rate, n_all, lane);
                return p.before_weight + p.weight * (count - p.before);
            };
            if (draw.top_k > 0 && draw.top_k < n) { n = draw.top_k; total = first_tokens(n); }
            int kept = n;
            if (draw.top_p < 1.0) {
                const double border = draw.top_p * total;
                const Place p = locate<F, kReach>(s, 0, border, top, draw.rate, n_all, lane);
                const double r = ceil((border - p.before_weight) / p.weight);      // tokens of the value with less than the border before them
                kept = min(kept, p.before + (r >= p.count ? p.count : r >= 1.0 ? (int)r : 1));
            }
            if (draw.min_p > 0.0) kept = min(kept, s_likely);
            kept = max(kept, 1);
            if (kept < n) total = first_tokens(kept);
            const double border = draw.uniform * total;
            Place p = locate<F, kPass>(s, 0, border, top, draw.rate, n_all, lane);
            const double r = floor((border - p.before_weight) / p.weight);
            int rank = r >= p.count ? p.count - 1 : r >= 1.0 ? (int)r : 0;
            if (p.before + rank >= kept) {                 // (rounding, or a number that is not below 1: the last of those kept)
                p = locate<F, kByCount>(s, kept, 0.0, top, draw.rate, n_all, lane);
                rank = kept - 1 - p.before;
            }
            const uint32_t word = word_at(p.seg, p.at);
            if (word == 0u && p.seg >= kHalf) rank += count_at(s, kHalf - 1, 63);      // -0 and +0 are one value
            if (lane == 0) {
                s_word = word;
                s_sign = p.seg < kHalf ? 0u : 0x8000u;
                s_rank = rank;
                put_draw(b, -1, log(p.weight / total), kept, out_tokens, out_logprobs, out_kept);
            }
        }
        __syncthreads();
        const uint32_t word = s_word, sign = word ? s_sign : 0u, care = word ? 0xFFFFu : 0x7FFFu;
        const int token = find_token<2>(row, mask, vocab, s_rank, [=](uint32_t h) { return (h & care) == (word | sign); }, s_part_count, &s_found, tid);
        if (tid == 0) out_tokens[b] = token;
        return;
    }
    // nothing to draw from: the first token of -inf, as for the arg max, or none
    const int token = find_token<2>(row, mask, vocab, 0, [=](uint32_t h) { return h == (F::kInf | 0x8000u); }, s_part_count, &s_found, tid);
    if (tid == 0) put_draw(b, token, token < 0 ? -(double)INFINITY : 0.0, token < 0 ? 0 : 1, out_tokens, out_logprobs, out_kept);
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
        const int cs = wave_scan_int(c[kPer - 1], lane);
        const unsigned long long ws = wave_scan_int(w[kPer - 1], lane);
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
    const dim3 grid(batch), block(kSampleBlock);
    if (type == kLogitBf16)
        hipLaunchKernelGGL(sample_counts_kernel<Bf16>, grid, block, 0, stream, static_cast<const uint16_t *>(logits), bitmask, vocab, row_stride,
                           n_words, rows, out_tokens, out_logprobs, out_kept);
    else if (type == kLogitF16)
        hipLaunchKernelGGL(sample_counts_kernel<F16>, grid, block, 0, stream, static_cast<const uint16_t *>(logits), bitmask, vocab, row_stride,
                           n_words, rows, out_tokens, out_logprobs, out_kept);
    else {
        int bits = 62;                          // the vocabulary's sum of weights stays below 2^63
        while (bits > 30 && ((int64_t)1 << (62 - bits)) < vocab) --bits;
        hipLaunchKernelGGL(sample_classes_kernel, grid, block, 0, stream, static_cast<const uint32_t *>(logits), bitmask, vocab, row_stride,
                           n_words, bits, rows, out_tokens, out_logprobs, out_kept);
    }
    return hipGetLastError();
}

}  // namespace pre3
