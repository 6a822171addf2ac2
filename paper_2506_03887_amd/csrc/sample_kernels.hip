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
#include "lanes.hpp"
#include "launch.hpp"
#include "rows.hpp"
#include "stream_access.hpp"

namespace pre3 {

namespace {


// What a row is drawn by.  A temperature that is not above zero decodes greedily (the draw from one token).
struct RowDraw {
    double rate, top_p, min_p, uniform;      // rate: 1 / temperature; top_p 1 and min_p 0: off
    int top_k;                               // 0: off
};
__device__ __forceinline__ double uniform_value(double x) {             // the same in every lane: kept in scalar registers
    const unsigned long long v = __builtin_bit_cast(unsigned long long, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32));
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ RowDraw row_draw(const SampleRows &rows, int b) {
    RowDraw d;
    const float t = rows.temperature ? rows.temperature[b] : 1.0f, u = rows.uniform[b];
    const float p = rows.top_p ? rows.top_p[b] : 1.0f, m = rows.min_p ? rows.min_p[b] : 0.0f;
    const int k = rows.top_k ? rows.top_k[b] : 0;
    const bool greedy = !(t > 0.0f);
    d.rate = uniform_value(greedy ? 1.0 : 1.0 / (double)t);
    d.top_k = __builtin_amdgcn_readfirstlane(greedy ? 1 : k > 0 ? k : 0);
    d.top_p = uniform_value(p < 1.0f ? (double)p : 1.0);  // (a NaN is off)
    d.min_p = uniform_value(m > 0.0f ? (double)m : 0.0);
    d.uniform = uniform_value(u > 0.0f ? (u < 1.0f ? (double)u : 1.0) : 0.0);
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
// fn(pattern, token) for every allowed token of a row, group of eight by group, groups of a thread kBlock apart.
template <int kBlock, int kBytes, class Fn>
__device__ __forceinline__ void each_allowed(const void *row, const uint8_t *mask, int vocab, int tid, Fn fn) {
    const int whole = vocab >> 3;
    for (int g = tid; g < whole; g += kBlock) {
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
template <int kBlock, int kBytes, class Hit>
__device__ int find_token(const void *row, const uint8_t *mask, int vocab, int rank, Hit hit, int *s_part, int *s_found, int tid) {
    const int lane = tid & 63, wave = tid >> 6, whole = vocab >> 3, groups = (vocab + 7) >> 3;
    const unsigned long long lanes_below = (1ull << lane) - 1ull;
    int base = 0;
    if (tid == 0) *s_found = -1;
    __syncthreads();
    for (int g0 = 0; g0 < groups; g0 += kBlock) {
        const int g = g0 + tid;
        uint32_t hits = 0u;
        if (g < groups) {
            const uint32_t mu = (mask ? mask[g] : 0xFFu) & (g < whole ? 0xFFu : (1u << (vocab & 7)) - 1u);
            if (mu != 0u) {
                uint32_t x[8];
                if (g < whole) load_group<kBytes>(row, g, x);
#pragma unroll
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
        for (int w = 0; w < kBlock / 64; ++w) {
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

// ------------------------------------------------------------------------------- rows of few candidates

__device__ __forceinline__ uint32_t falling_key(float x) {                  // ascending keys: descending numbers; -0 as +0
    const uint32_t bits = __float_as_uint(x + 0.0f);
    return bits ^ (~(uint32_t)((int)bits >> 31) & 0x7FFFFFFFu);
}
__device__ __forceinline__ float of_falling_key(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key : key ^ 0x7FFFFFFFu); }
constexpr uint32_t kKeyPosInf = 0x007FFFFFu, kKeyNegInf = 0xFF800000u;      // NaNs lie outside
__device__ __forceinline__ bool is_candidate(uint32_t key) { return key - kKeyPosInf < kKeyNegInf - kKeyPosInf; }

// Up to a thousand candidates are sorted, key above id, and everything is a place among them.  The bitonic network's exchanges of
// up to 32 places run between the lanes of a wave, the others through LDS.
template <int kBlock>
struct Sorted {
    unsigned long long entry[kBlock];
    double upto[kBlock];                       // weights summed, the place included
    double part[kBlock / 64];
    int likely;
};
constexpr unsigned long long kNoEntry = ~0ull;
__device__ __forceinline__ unsigned long long exchanged(unsigned long long mine, unsigned long long other, int j, int k, int place) {
    const bool smaller = ((place & j) == 0) == ((place & k) == 0);           // this place keeps the smaller of the two
    return (other < mine) == smaller ? other : mine;
}
__device__ __forceinline__ unsigned long long exchanged_in_wave(unsigned long long mine, int j, int k, int place) {
    const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)mine, j), hi = (uint32_t)__shfl_xor((int)(uint32_t)(mine >> 32), j);
    return exchanged(mine, (unsigned long long)hi << 32 | lo, j, k, place);
}
template <int kBlock>
__device__ __forceinline__ unsigned long long sorted_entry(unsigned long long mine, int size, unsigned long long *s_entry, int tid) {
    for (int k = 2; k <= size; k *= 2) {
        for (int j = k / 2; j > 0; j /= 2) {
            if (j < 64) {
                mine = exchanged_in_wave(mine, j, k, tid);
            } else {
                lds_barrier();
                s_entry[tid] = mine;
                lds_barrier();
                mine = exchanged(mine, s_entry[tid ^ j], j, k, tid);
            }
        }
    }
    return mine;
}
// The draw from n >= 1 candidates, each thread's entry a key above an id or kNoEntry, the first `size` (a power of two) threads' ones all there are.
template <int kBlock>
__device__ __forceinline__ void draw_sorted(Sorted<kBlock> &s, unsigned long long mine, int size, int n, const RowDraw &draw, int b, int32_t *out_tokens, float *out_logprobs,
                                            int32_t *out_kept, int tid) {
    mine = sorted_entry<kBlock>(mine, size, s.entry, tid);
    lds_barrier();
    s.entry[tid] = mine;
    if (tid == 0) s.likely = 0;
    lds_barrier();
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const double top = (double)of_falling_key((uint32_t)(s.entry[0] >> 32));
    const double w = tid < n ? draw_weight((double)of_falling_key((uint32_t)(mine >> 32)), top, draw.rate) : 0.0;
    double upto = wave_scan(w);
    if (lane == 63) s.part[wave] = upto;
    if (draw.min_p > 0.0) {
        const unsigned long long likely = __ballot(tid < n && w >= draw.min_p);
        if (lane == 0 && likely) atomicAdd(&s.likely, __popcll(likely));
    }
    lds_barrier();
    for (int v = 0; v < wave; ++v) upto += s.part[v];
    s.upto[tid] = upto;
    lds_barrier();
    if (wave != 0) return;
    // the first place whose sum is above (kPass: above, else at least) the border
    auto first_place = [&](double border, bool pass, int last) {
        int lo = 0, hi = last;                 // (the last one if rounding leaves none)
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (pass ? s.upto[mid] > border : s.upto[mid] >= border) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    };
    int kept = draw.top_k > 0 && draw.top_k < n ? draw.top_k : n;
    if (draw.top_p < 1.0) {
        const int through = first_place(draw.top_p * s.upto[kept - 1], false, kept - 1) + 1;
        kept = through < kept ? through : kept;
    }
    if (draw.min_p > 0.0) kept = min(kept, max(s.likely, 1));
    const double total = s.upto[kept - 1];
    const int at = first_place(draw.uniform * total, true, kept - 1);
    const unsigned long long entry = s.entry[at];
    if (lane == 0)
        put_draw(b, (int)(uint32_t)entry, log(draw_weight((double)of_falling_key((uint32_t)(entry >> 32)), top, draw.rate) / total), kept, out_tokens, out_logprobs, out_kept);
}

// The draw by one wave from up to 64 allowed tokens, each lane's key above its id (kNoEntry: none, or its logit is a NaN).
__device__ __forceinline__ void draw_by_wave(unsigned long long mine, const RowDraw &draw, int b, int32_t *out_tokens, float *out_logprobs, int32_t *out_kept, int lane) {
    for (int k = 2; k <= 64; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) mine = exchanged_in_wave(mine, j, k, lane);
    const uint32_t key = (uint32_t)(mine >> 32);
    const int n = __popcll(__ballot(is_candidate(key)));
    if (n == 0) {                              // the first token of -inf, or none
        const unsigned long long first = from_lane(mine, 0);
        const bool none = first == kNoEntry;
        if (lane == 0) put_draw(b, none ? -1 : (int)(uint32_t)first, none ? -(double)INFINITY : 0.0, none ? 0 : 1, out_tokens, out_logprobs, out_kept);
        return;
    }
    const double w = lane < n ? draw_weight((double)of_falling_key(key), (double)of_falling_key(from_lane(key, 0)), draw.rate) : 0.0, upto = wave_scan(w);
    // the first place for which it holds, or the last one kept
    int kept = draw.top_k > 0 && draw.top_k < n ? draw.top_k : n;
    auto first_place = [&](bool holds) {
        const unsigned long long has = __ballot(holds && lane < kept);
        return has ? __ffsll(has) - 1 : kept - 1;
    };
    if (draw.top_p < 1.0) {
        const double border = draw.top_p * from_lane(upto, kept - 1);
        kept = first_place(upto >= border) + 1;
    }
    if (draw.min_p > 0.0) kept = min(kept, max(__popcll(__ballot(lane < n && w >= draw.min_p)), 1));
    const double total = from_lane(upto, kept - 1), border = draw.uniform * total;
    const int at = first_place(upto > border);
    if (lane == at) put_draw(b, (int)(uint32_t)mine, log(w / total), kept, out_tokens, out_logprobs, out_kept);
}

// ------------------------------------------------------------------------------- logits of 16 bits

// A row of 16-bit logits has at most 65,536 different values: how many tokens have each is all that the draw needs, exactly, and
// weights are computed once for a value, in 64 bits.  Counts lie in LDS, 16 bits for a value, the two signs of a magnitude in one word
// (word = pattern without the sign), so that a token is one add without a return and a pattern needs no reordering.
// The order descends through the positive words, then ascends through the negative ones: 256 segments of 256 values each.
struct Bf16 {
    static constexpr uint32_t kInf = 0x7F80u;
    __device__ static double value(uint32_t h) { return (double)__uint_as_float(h << 16); }
};
struct F16 {
    static constexpr uint32_t kInf = 0x7C00u;
    __device__ static double value(uint32_t h) { return (double)(float)__builtin_bit_cast(_Float16, (uint16_t)h); }
};
constexpr int kCountBlock = 1024, kCountWaves = kCountBlock / 64;
constexpr int kWords = 32768, kSegmentWords = 256, kHalf = kWords / kSegmentWords, kSegments = 2 * kHalf;
constexpr int kMaxHeavy = 8;                              // segments that can hold 65,536 tokens or more of a row

__device__ __forceinline__ int segment_of(uint32_t word, uint32_t sign) { return sign ? kHalf + (int)(word / kSegmentWords) : kHalf - 1 - (int)(word / kSegmentWords); }
__device__ __forceinline__ uint32_t word_at(int seg, int at) {
    return seg < kHalf ? (uint32_t)(kHalf - 1 - seg) * kSegmentWords + (kSegmentWords - 1 - at) : (uint32_t)(seg - kHalf) * kSegmentWords + at;
}

struct CountTables {
    uint32_t count[kWords];
    __align__(16) double weight[kSegments];               // of every segment
    __align__(16) int tokens[kSegments];
    double sum[64];                                       // through the order, before every fourth segment; all of them
    int upto[64];
    double total;
    int n_all;
    uint32_t heavy[kMaxHeavy][kSegmentWords];             // counts that 16 bits do not hold, by place in the segment
    int heavy_segment[kMaxHeavy], n_heavy;
};

// A wave looks at a segment with four neighbouring values a lane, in the order of the draw: how many tokens have each (none where the
// value is a NaN or -inf), and a token's weight.
struct Four { int count[4]; double weight[4]; };
template <class F>
__device__ __forceinline__ void counts_of(const CountTables &s, int seg, int n_heavy, int lane, Four &f) {
    const uint32_t low = min(word_at(seg, lane * 4), word_at(seg, lane * 4 + 3));
    const uint4 x = *reinterpret_cast<const uint4 *>(s.count + low);
    if (seg < kHalf) {
        f.count[0] = x.w & 0xFFFFu; f.count[1] = x.z & 0xFFFFu; f.count[2] = x.y & 0xFFFFu; f.count[3] = x.x & 0xFFFFu;
    } else {
        f.count[0] = x.x >> 16; f.count[1] = x.y >> 16; f.count[2] = x.z >> 16; f.count[3] = x.w >> 16;
    }
    for (int i = 0; i < n_heavy; ++i) {
        if (s.heavy_segment[i] == seg) {
            for (int k = 0; k < 4; ++k) f.count[k] = (int)s.heavy[i][lane * 4 + k];
            break;
        }
        // a positive count beyond 16 bits has carried into the negative one
        if (seg >= kHalf && s.heavy_segment[i] == segment_of(low, 0))
            for (int k = 0; k < 4; ++k) f.count[k] = (f.count[k] - (int)(s.heavy[i][kSegmentWords - 1 - (lane * 4 + k)] >> 16)) & 0xFFFF;
    }
    if (low >= F::kInf) {                                 // (the first word of a lane: +inf is its last place, -inf does not count)
        f.count[0] = f.count[1] = f.count[2] = 0;
        if (low > F::kInf || seg >= kHalf) f.count[3] = 0;
    }
}
// The row's maximum and where it stands.
struct Top { double value; int seg, at; };
// Neighbours of a lane lie one step of their octave apart, so that each weight is the one before times the same factor: two exponentials
// for four.  Where the maximum itself is one of the four it is what the others count from.
template <class F>
__device__ __forceinline__ void weights_of(int seg, const Top &top, double rate, int lane, Four &f) {
    const uint32_t sign = seg < kHalf ? 0u : 0x8000u, word = word_at(seg, lane * 4);
    const double value = F::value(word | sign), next = F::value(word_at(seg, lane * 4 + 1) | sign);
    const int behind = seg == top.seg && lane == top.at >> 2 ? top.at & 3 : 0;
    const double factor = exp_of_negative((next - value) * rate);
    double w = exp_of_negative((fmin(value, top.value) - top.value) * rate);
    if (word >= F::kInf) w = 1.0;                         // (+inf is the maximum where it occurs)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (k > behind && word < F::kInf) w *= factor;
        f.weight[k] = w;
    }
}
__device__ __forceinline__ int tokens_of(const Four &f) { return (f.count[0] + f.count[1]) + (f.count[2] + f.count[3]); }
__device__ __forceinline__ double weight_of(const Four &f) {
    return fma((double)f.count[3], f.weight[3], fma((double)f.count[2], f.weight[2], fma((double)f.count[1], f.weight[1], (double)f.count[0] * f.weight[0])));
}

// A place in the order: the value with the token searched for, what lies before the value, and its number of tokens.
struct Place {
    int seg, at, before, count;
    double before_weight, weight;                         // weight: of one of its tokens
};
// What a search looks for: the first value up to and including which the order has more than `limit` tokens, or weight.
struct Sought { bool tokens; double limit; };
__device__ __forceinline__ Sought first_tokens(int n) { return {true, n - 0.5}; }
__device__ __forceinline__ Sought weight_above(double border) { return {false, border}; }
__device__ __forceinline__ Sought weight_of_at_least(double border) {      // above the number before it
    return {false, border > 0.0 ? __builtin_bit_cast(double, __builtin_bit_cast(unsigned long long, border) - 1ull) : -1.0};
}
// By one wave.  A limit that rounding puts behind the last value gives the last one.
template <class F>
__device__ __forceinline__ Place locate(const CountTables &s, Sought sought, const Top &top, double rate, int n_heavy, int lane) {
    // every lane walks through its own four (behind `c` and `w`); the first lane that finds enough has the place
    struct Step { int lane, at, before; double before_weight; };
    auto step = [&](const int *tokens, const double *weights, int c0, double w0) {
        int c[5] = {c0};
        double w[5] = {w0};
#pragma unroll
        for (int k = 0; k < 4; ++k) { c[k + 1] = c[k] + tokens[k]; w[k + 1] = w[k] + weights[k]; }
        uint32_t enough;
        unsigned long long has;
        for (;;) {
            enough = 0u;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const double x = sought.tokens ? (double)c[k + 1] : w[k + 1];
                enough |= (x > sought.limit && tokens[k] != 0 ? 1u : 0u) << k;
            }
            has = __ballot(enough != 0u);
            if (has) break;
            sought = first_tokens(from_lane(c[4], 63));    // rounding: the last token there is
        }
        const int at = __ffs(enough) - 1;
        Step r;
        r.lane = __builtin_amdgcn_readfirstlane(__ffsll(has) - 1);
        r.at = from_lane(at, r.lane);
        r.before = from_lane(at == 0 ? c[0] : at == 1 ? c[1] : at == 2 ? c[2] : c[3], r.lane);
        r.before_weight = from_lane(at == 0 ? w[0] : at == 1 ? w[1] : at == 2 ? w[2] : w[3], r.lane);
        return r;
    };
    const int4 t4 = *reinterpret_cast<const int4 *>(s.tokens + lane * 4);
    const int tokens[4] = {t4.x, t4.y, t4.z, t4.w};
    const double weights[4] = {s.weight[lane * 4], s.weight[lane * 4 + 1], s.weight[lane * 4 + 2], s.weight[lane * 4 + 3]};
    const Step segment = step(tokens, weights, s.upto[lane], s.sum[lane]);
    Place p;
    p.seg = segment.lane * 4 + segment.at;
    Four f;
    counts_of<F>(s, p.seg, n_heavy, lane, f);
    weights_of<F>(p.seg, top, rate, lane, f);
    double all[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) all[k] = f.weight[k] * f.count[k];
    const int c = tokens_of(f);
    const double w = (all[0] + all[1]) + (all[2] + all[3]);
    const Step value = step(f.count, all, wave_scan(c) - c + segment.before, wave_scan(w) - w + segment.before_weight);
    p.at = value.lane * 4 + value.at;
    p.before = value.before;
    p.before_weight = value.before_weight;
    p.count = from_lane(value.at == 0 ? f.count[0] : value.at == 1 ? f.count[1] : value.at == 2 ? f.count[2] : f.count[3], value.lane);
    p.weight = from_lane(value.at == 0 ? f.weight[0] : value.at == 1 ? f.weight[1] : value.at == 2 ? f.weight[2] : f.weight[3], value.lane);
    return p;
}

// Counts of 16 bits have overflowed: segments are counted in 32 bits and the heavy ones value by value.  A call of its own.
__device__ __noinline__ void count_heavy(CountTables &s, const uint16_t *row, const uint8_t *mask, int vocab) {
    const int tid = threadIdx.x;
    for (int i = tid; i < kSegments; i += kCountBlock) s.tokens[i] = 0;
    __syncthreads();
    each_allowed<kCountBlock, 2>(row, mask, vocab, tid, [&](uint32_t h, int) { atomicAdd(&s.tokens[segment_of(h & 0x7FFFu, h >> 15)], 1); });
    __syncthreads();
    if (tid == 0) {
        int n = 0;
        for (int i = 0; i < kSegments && n < kMaxHeavy; ++i)
            if (s.tokens[i] > 0xFFFF) s.heavy_segment[n++] = i;
        s.n_heavy = n;
    }
    __syncthreads();
    const int n_heavy = s.n_heavy;
    for (int i = tid; i < n_heavy * kSegmentWords; i += kCountBlock) s.heavy[i / kSegmentWords][i % kSegmentWords] = 0u;
    for (int i = tid; i < kSegments; i += kCountBlock) s.tokens[i] = 0;
    __syncthreads();
    each_allowed<kCountBlock, 2>(row, mask, vocab, tid, [&](uint32_t h, int) {
        const int seg = segment_of(h & 0x7FFFu, h >> 15), at = (int)(h % kSegmentWords);
        for (int i = 0; i < n_heavy; ++i)
            if (s.heavy_segment[i] == seg) atomicAdd(&s.heavy[i][seg < kHalf ? kSegmentWords - 1 - at : at], 1u);
    });
    __syncthreads();
}

// find_token for the tokens whose pattern is the given one in the bits `care`.  A call of its own: rows that come here are rare.
__device__ __noinline__ int find_pattern(const uint16_t *row, const uint8_t *mask, int vocab, int rank, uint32_t pattern, uint32_t care, int *s_part, int *s_found) {
    return find_token<kCountBlock, 2>(row, mask, vocab, rank, [=](uint32_t h) { return ((h ^ pattern) & care & 0xFFFFu) == 0u; }, s_part, s_found, threadIdx.x);
}

// What wave 0 has drawn: the pattern (0 stands for both zeros), how many tokens have it, the token's rank among them by id, its
// weight, and the tokens kept with their weight.
struct Drawn { uint32_t word, sign; int equal, rank, kept; double weight, total; };

// By wave 0: what is kept, and the draw.  (One search after the other in a loop, so that its code is there once: a block runs
// through it once, and fetching code takes longer than running it.)
template <class F>
__device__ __forceinline__ Drawn draw_from_counts(const CountTables &s, const RowDraw &draw, const Top &top, int likely, int n_heavy, int lane) {
    Drawn d;
    d.kept = s.n_all;
    d.total = s.total;
    enum Step { kTopK, kTopP, kMinP, kDraw, kLastKept };
    for (int step = kTopK; step <= kLastKept; ++step) {
        int n = step == kTopK ? draw.top_k : max(likely, 1);
        if (step == kTopK && !(draw.top_k > 0 && draw.top_k < d.kept)) continue;
        if (step == kTopP && !(draw.top_p < 1.0)) continue;
        if (step == kMinP && !(draw.min_p > 0.0 && n < d.kept)) continue;
        if (step == kLastKept) n = d.kept;
        const double border = (step == kTopP ? draw.top_p : draw.uniform) * d.total;
        const Place p = locate<F>(s, step == kTopP ? weight_of_at_least(border) : step == kDraw ? weight_above(border) : first_tokens(n), top, draw.rate, n_heavy, lane);
        if (step == kTopP) {                               // tokens of the value with less than the border before them
            const double r = ceil((border - p.before_weight) / p.weight);
            n = p.before + (r >= p.count ? p.count : r >= 1.0 ? (int)r : 1);
        }
        if (step < kDraw) {
            if (n < d.kept) { d.kept = n; d.total = p.before_weight + p.weight * (n - p.before); }
            continue;
        }
        const double r = floor((border - p.before_weight) / p.weight);
        d.rank = step == kLastKept ? d.kept - 1 - p.before : r >= p.count ? p.count - 1 : r >= 1.0 ? (int)r : 0;
        if (step == kDraw && p.before + d.rank >= d.kept) continue;        // (rounding, or a number that is not below 1: the last of those kept)
        d.word = word_at(p.seg, p.at);
        d.sign = p.seg < kHalf ? 0u : 0x8000u;
        d.equal = p.count;
        d.weight = p.weight;
        break;
    }
    if (d.word == 0u) {                                    // -0 and +0 are one value
        Four f;
        counts_of<F>(s, d.sign ? kHalf - 1 : kHalf, n_heavy, lane, f);
        const int others = d.sign ? from_lane(f.count[3], 63) : from_lane(f.count[0], 0);
        if (d.sign) d.rank += others;
        d.equal += others;
        d.sign = 0u;
    }
    return d;
}

// Two tokens of 16 bits in a register: which halves of x are equal to those of `pair` where `care` has bits, as zero halves.
__device__ __forceinline__ uint32_t differing(uint32_t x, uint32_t pair, uint32_t care) { return (x ^ pair) & care; }
typedef unsigned short PackedU16 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t packed_min(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(PackedU16, a), __builtin_bit_cast(PackedU16, b)));
}
__device__ __forceinline__ uint32_t packed_signs(uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(PackedU16, x) >> 15); }

// One block a row, kG groups of eight tokens a thread; a row of more than a block's kG * 8,192 tokens (kMany) goes through in chunks and is
// read again for the token's id.
template <class F, int kG, bool kMany>
__global__ __launch_bounds__(kCountBlock) void sample_counts_kernel(const uint16_t *__restrict__ logits, const uint32_t *__restrict__ bitmask,
                                                                    int vocab, int64_t row_stride, int n_words, SampleRows rows,
                                                                    int32_t *__restrict__ out_tokens, float *__restrict__ out_logprobs,
                                                                    int32_t *__restrict__ out_kept) {
    constexpr int kAhead = kG < 3 ? kG : 3, kLook = kHalf / kCountWaves;                  // groups in flight; looks at the words of a segment a wave
    constexpr int kKept = kG < 12 ? kG : 12;              // groups that stay in registers through the draw (all 20: 45 registers spilled)
    __shared__ __align__(16) CountTables s;
    struct Group { uint4 x; uint32_t allowed; int at; };
    __shared__ Group s_rest;
    __shared__ uint2 s_ones[16];                          // four mask bits -> 1 or 0 in the halves of two registers
    __shared__ uint16_t s_busy[kSegments];                // segments that have tokens
    __shared__ int s_first, s_likely, s_seen, s_n_busy, s_listed, s_equal, s_part[kCountWaves], s_id[kCountBlock];
    __shared__ Drawn s_drawn;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
    const uint16_t *row = logits + (size_t)b * row_stride;
    const uint8_t *mask = bitmask ? reinterpret_cast<const uint8_t *>(bitmask + (size_t)b * n_words) : nullptr;
    const int whole = vocab >> 3, rest = vocab & 7, chunks = kMany ? (whole + kG * kCountBlock - 1) / (kG * kCountBlock) : 1;
    uint4 v[kG];
    uint32_t packed[(kG + 3) / 4];                         // mask bytes of the groups, 0 behind the row
    auto first_group = [&](int chunk) { return chunk * (kG * kCountBlock) + tid; };         // of a thread; its others are kCountBlock apart
    auto load_masks = [&](int chunk) {
        const int first = first_group(chunk);
        uint32_t m[kG];
#pragma unroll
        for (int u = 0; u < kG; ++u) m[u] = mask ? mask[min(first + u * kCountBlock, max(whole - 1, 0))] : 0xFFu;
#pragma unroll
        for (int u = 0; u < kG; ++u) packed[u / 4] = (u & 3 ? packed[u / 4] : 0u) | (first + u * kCountBlock < whole ? m[u] : 0u) << (8 * (u & 3));
    };
    auto load = [&](int chunk, int u) {
        uint32_t at = (uint32_t)first_group(chunk) * 16u;
        asm volatile("" : "+v"(at));                       // (each load finds its place anew: the places of all would take the groups' registers)
        at = min(at + (uint32_t)(u * kCountBlock) * 16u, (uint32_t)(whole - 1) * 16u);
        // (once the mask is there, a group of which nothing is allowed is not fetched: its lane asks for its first group again)
        if (u >= kAhead && ((packed[u / 4] >> (8 * (u & 3))) & 0xFFu) == 0u) at = 0u;
        v[u] = stream_load_at(row, at);
    };
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
    // (1) counts; a row of which the mask allows at most 64 tokens is one wave's instead
    constexpr int kMaskWords = (kG + 3) / 4;               // of a thread
    const bool may_be_few = !kMany && mask != nullptr;
    uint32_t words[kMaskWords];
    if (may_be_few) {
#pragma unroll
        for (int i = 0; i < kMaskWords; ++i) words[i] = reinterpret_cast<const uint32_t *>(mask)[min(tid + i * kCountBlock, n_words - 1)];
    }
    load_masks(0);
    load_all(0, 0, kAhead);
    if (rest && tid == 0) {                                // the last group, which is not whole
        uint32_t x[4] = {0u, 0u, 0u, 0u};
        for (int k = 0; k < rest; ++k) x[k >> 1] |= (uint32_t)row[whole * 8 + k] << (16 * (k & 1));
        s_rest.x = make_uint4(x[0], x[1], x[2], x[3]);
        s_rest.allowed = (mask ? mask[whole] : 0xFFu) & ((1u << rest) - 1u);
    }
    const RowDraw draw = row_draw(rows, b);
    for (int i = tid; i < kWords / 4; i += kCountBlock) reinterpret_cast<uint4 *>(s.count)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid < kSegments) { s.tokens[tid] = 0; s.weight[tid] = 0.0; }
    if (tid < 16) s_ones[tid] = make_uint2((tid & 1) | (tid & 2) << 15, (tid >> 2 & 1) | (tid >> 2 & 2) << 15);
    if (tid == 0) { s.n_heavy = 0; s_first = kSegments; s_likely = 0; s_seen = 0; s_n_busy = 0; s_listed = 0; s_equal = 0; }
#pragma unroll
    for (int i = 0; i < (kG + 3) / 4; ++i) asm volatile("" : "+v"(packed[i]));             // (packed before the groups take the registers)
    int allowed = 0;
    if (may_be_few) {
#pragma unroll
        for (int i = 0; i < kMaskWords; ++i) {
            const int at = tid + i * kCountBlock;
            if (at >= n_words) words[i] = 0u;
            if (at == n_words - 1 && (vocab & 31)) words[i] &= (1u << (vocab & 31)) - 1u;
            allowed += __popc(words[i]);
        }
        const int sum = wave_sum(allowed);
        if (lane == 0) s_part[wave] = sum;
    }
    lds_barrier();
    if (may_be_few && wave_sum(lane < kCountWaves ? s_part[lane] : 0) <= 64) {
        if (allowed != 0) {
            int to = atomicAdd(&s_listed, allowed);
#pragma unroll
            for (int i = 0; i < kMaskWords; ++i)
                for (uint32_t left = words[i]; left; left &= left - 1u) s_id[to++] = (tid + i * kCountBlock) * 32 + __ffs(left) - 1;
        }
        lds_barrier();
        if (wave != 0) return;
        const int token = lane < s_listed ? s_id[lane] : -1;
        const float x = token < 0 ? __uint_as_float(0x7FC00000u) : (float)F::value(row[token]);
        draw_by_wave(x == x ? (unsigned long long)falling_key(x) << 32 | (uint32_t)token : kNoEntry, draw, b, out_tokens, out_logprobs, out_kept, lane);
        return;
    }
    if (rest && tid == 0) count_group(s_rest.x, s_rest.allowed);
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
    lds_barrier();
    // (2) the segments with tokens, the first of them, and whether the counts are whole
    uint32_t counted = 0u, with_tokens = 0u;               // bit i, 16 + i: the positive, the negative segment of the words looked at
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
        const uint32_t at = (uint32_t)(wave + i * kCountWaves) * kSegmentWords + (uint32_t)lane * 4u;
        const uint4 c = *reinterpret_cast<const uint4 *>(s.count + at);
        counted = __builtin_amdgcn_sad_u16(c.x, 0u, __builtin_amdgcn_sad_u16(c.y, 0u, __builtin_amdgcn_sad_u16(c.z, 0u, __builtin_amdgcn_sad_u16(c.w, 0u, counted))));
        uint32_t any = c.x | c.y | c.z | c.w;
        static_assert(F::kInf / kSegmentWords >= (kLook - 1) * kCountWaves, "infinities and NaNs in the last look only");
        if (i == kLook - 1 && at >= F::kInf) any = at == F::kInf ? c.x & 0xFFFFu : 0u;     // +inf, no -inf, no NaNs
        if (__ballot((any & 0xFFFFu) != 0u) != 0ull) with_tokens |= 1u << i;
        if (__ballot(any > 0xFFFFu) != 0ull) with_tokens |= 0x10000u << i;
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    auto add_busy = [&](bool mine, int seg) {              // a segment a lane
        const unsigned long long has = __ballot(mine);
        if (has == 0ull) return;
        int slot = 0;
        if (lane == 0) slot = atomicAdd(&s_n_busy, __popcll(has));
        slot = __builtin_amdgcn_readfirstlane(slot);
        if (mine) {
            s_busy[slot + __popcll(has & ((1ull << lane) - 1ull))] = (uint16_t)seg;
            atomicMin(&s_first, seg);
        }
    };
    add_busy((with_tokens >> (lane & 31)) & (lane < 32 ? 1u : 0u), segment_of((uint32_t)(wave + (lane & 15) * kCountWaves) * kSegmentWords, lane & 16));
    if (vocab > 0xFFFF) {
        // Counts beyond 16 bits carry or vanish, and the sum tells.
        const int missing = wave_sum((int)(seen - counted));
        if (lane == 0 && missing != 0) atomicAdd(&s_seen, missing);
    }
    lds_barrier();
    if (s_seen != 0) {
        count_heavy(s, row, mask, vocab);
        if (!kMany) {                                      // (again: they do not stay in registers over a call)
            load_masks(0);
            load_all(0, 0, kG);
        }
        if (tid == 0) { s_n_busy = 0; s_first = kSegments; }
        lds_barrier();
        for (int j = wave; j < kSegments; j += kCountWaves) {
            Four f;
            counts_of<F>(s, j, s.n_heavy, lane, f);
            add_busy(__any(tokens_of(f) != 0) && lane == 0, j);
        }
        lds_barrier();
    }
    const int n_heavy = s.n_heavy;
    const int first = s_first;
    if (first == kSegments) {
        // nothing to draw from: the first token of -inf, as for the arg max, or none
        const int token = find_pattern(row, mask, vocab, 0, F::kInf | 0x8000u, 0xFFFFu, s_part, &s_seen);
        if (tid == 0) put_draw(b, token, token < 0 ? -(double)INFINITY : 0.0, token < 0 ? 0 : 1, out_tokens, out_logprobs, out_kept);
        return;
    }
    // (3) every segment's count and weight
    Top top;
    {
        Four f;
        counts_of<F>(s, first, n_heavy, lane, f);
        const int from = __builtin_amdgcn_readfirstlane(__ffsll(__ballot(tokens_of(f) != 0)) - 1), k = f.count[0] ? 0 : f.count[1] ? 1 : f.count[2] ? 2 : 3;
        top.seg = first;
        top.at = from * 4 + from_lane(k, from);
        top.value = F::value(word_at(first, top.at) | (first < kHalf ? 0u : 0x8000u));
    }
    const int n_busy = s_n_busy;
    int likely = 0;
    for (int i = wave; i < n_busy; i += kCountWaves) {
        const int seg = __builtin_amdgcn_readfirstlane(s_busy[i]);
        Four f;
        counts_of<F>(s, seg, n_heavy, lane, f);
        weights_of<F>(seg, top, draw.rate, lane, f);
        if (draw.min_p > 0.0) {
#pragma unroll
            for (int k = 0; k < 4; ++k) likely += f.weight[k] >= draw.min_p ? f.count[k] : 0;
        }
        const int tokens = wave_scan(tokens_of(f));
        const double weight = wave_scan(weight_of(f));
        if (lane == 63) { s.tokens[seg] = tokens; s.weight[seg] = weight; }
    }
    if (draw.min_p > 0.0) {
        likely = wave_sum(likely);
        if (lane == 0) atomicAdd(&s_likely, likely);
    }
    lds_barrier();
    // (4) the draw, by wave 0
    if (wave == 0) {
        const int tokens = (s.tokens[lane * 4] + s.tokens[lane * 4 + 1]) + (s.tokens[lane * 4 + 2] + s.tokens[lane * 4 + 3]), upto = wave_scan(tokens);
        const double weight = (s.weight[lane * 4] + s.weight[lane * 4 + 1]) + (s.weight[lane * 4 + 2] + s.weight[lane * 4 + 3]), sum = wave_scan(weight);
        s.upto[lane] = upto - tokens;
        s.sum[lane] = sum - weight;
        if (lane == 63) { s.n_all = upto; s.total = sum; }
        wave_exchange();
        const Drawn d = draw_from_counts<F>(s, draw, top, s_likely, n_heavy, lane);
        if (lane == 0) s_drawn = d;
    }
    if (!kMany) load_all(0, kKept, kG);                    // (the other waves' are there by the time that the draw is)
    lds_barrier();
    // (5) the token's id: number `rank` among the allowed tokens with the pattern, by ascending id
    const uint32_t word = s_drawn.word, pattern = word | s_drawn.sign, care = word ? 0xFFFFFFFFu : 0x7FFF7FFFu, pair = pattern | pattern << 16;
    const int rank = s_drawn.rank, equal = s_drawn.equal;
    if (tid == 0) {
        if (out_logprobs) out_logprobs[b] = (float)log(s_drawn.weight / s_drawn.total);
        if (out_kept) out_kept[b] = s_drawn.kept;
    }
    // groups with such a token, masked or not, into a list (where the counts were); its allowed ones by id into another
    constexpr int kGroupList = kWords * 4 / sizeof(Group);
    Group *listed = reinterpret_cast<Group *>(s.count);
    auto least_of = [&](uint4 group) {                     // a half is zero where one of four tokens is equal
        return packed_min(packed_min(differing(group.x, pair, care), differing(group.y, pair, care)),
                          packed_min(differing(group.z, pair, care), differing(group.w, pair, care)));
    };
    auto some_equal = [](uint32_t least) { return (least & 0xFFFFu) == 0u || least < 0x10000u; };
    auto list_group = [&](uint4 group, uint32_t a, int at) {
        if (a == 0u || !some_equal(least_of(group))) return;
        const int i = atomicAdd(&s_listed, 1);
        if (i < kGroupList) listed[i] = {group, a, at};
    };
    if (equal <= kCountBlock) {
        for (int chunk = 0; chunk < chunks; ++chunk) {
            if (kMany) {
                load_masks(chunk);
                load_all(chunk, 0, kG);
            }
            uint32_t least = 0xFFFFFFFFu;
#pragma unroll
            for (int u = 0; u < kG; ++u) least = packed_min(least, least_of(v[u]));
            if (!__any(some_equal(least))) continue;       // (most waves, where most is allowed)
            int first = first_group(chunk);
            asm volatile("" : "+v"(first));                // (else the groups' numbers are kept from the loads on, in registers that are not there)
#pragma unroll
            for (int u = 0; u < kG; ++u) list_group(v[u], (packed[u / 4] >> (8 * (u & 3))) & 0xFFu, first + u * kCountBlock);
        }
        if (rest && tid == 0) list_group(s_rest.x, s_rest.allowed, whole);
    }
    lds_barrier();
    const int n_listed = s_listed;
    if (equal > kCountBlock || n_listed > kGroupList) {   // the lists do not hold them
        const int token = find_pattern(row, mask, vocab, rank, pattern, care, s_part, &s_seen);
        if (tid == 0) out_tokens[b] = token;
        return;
    }
    for (int i = tid; i < n_listed * 8; i += kCountBlock) {
        const Group &g = listed[i >> 3];
        const uint32_t x = reinterpret_cast<const uint16_t *>(&g.x)[i & 7];
        if (((g.allowed >> (i & 7)) & 1u) && ((x ^ pattern) & care & 0xFFFFu) == 0u) {
            const int id = g.at * 8 + (i & 7);
            if (equal == 1) out_tokens[b] = id;
            else s_id[atomicAdd(&s_equal, 1)] = id;
        }
    }
    if (equal == 1) return;
    lds_barrier();
    if (tid < equal) {
        const int id = s_id[tid];
        int smaller = 0;
        for (int i = 0; i < equal; ++i) smaller += s_id[i] < id ? 1 : 0;
        if (smaller == rank) out_tokens[b] = id;
    }
}

template <class F>
void launch_counts(const uint16_t *logits, const uint32_t *bitmask, int batch, int vocab, int64_t row_stride, int n_words, const SampleRows &rows,
                   int32_t *out_tokens, float *out_logprobs, int32_t *out_kept, hipStream_t stream) {
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(batch), dim3(kCountBlock), 0, stream, logits, bitmask, vocab, row_stride, n_words, rows, out_tokens,
                           out_logprobs, out_kept);
    };
    const int rounds = (vocab + kCountBlock * 8 - 1) / (kCountBlock * 8);
    if (rounds <= 1) go(sample_counts_kernel<F, 1, false>);
    else if (rounds <= 4) go(sample_counts_kernel<F, 4, false>);
    else if (rounds <= 8) go(sample_counts_kernel<F, 8, false>);
    else if (rounds <= 12) go(sample_counts_kernel<F, 12, false>);
    else if (rounds <= 16) go(sample_counts_kernel<F, 16, false>);
    else if (rounds <= 20) go(sample_counts_kernel<F, 20, false>);
    else go(sample_counts_kernel<F, 8, true>);
}

// ------------------------------------------------------------------------------- vocabularies of few tokens

// Vocabularies of up to kBlock tokens.
template <int kBlock, class F>
__global__ __launch_bounds__(kBlock) void sample_sorted_kernel(const typename F::Stored *__restrict__ logits, const uint32_t *__restrict__ bitmask, int vocab, int64_t row_stride,
                                                              int n_words, SampleRows rows, int32_t *__restrict__ out_tokens, float *__restrict__ out_logprobs,
                                                              int32_t *__restrict__ out_kept) {
    __shared__ Sorted<kBlock> s;
    __shared__ int s_n, s_neg_inf;
    const int tid = threadIdx.x, b = blockIdx.x;
    const Row<F> row = {logits + (size_t)b * row_stride, bitmask ? bitmask + (size_t)b * n_words : nullptr, vocab};
    if (tid == 0) { s_n = 0; s_neg_inf = vocab; }
    const bool allowed = tid < vocab && row.allows(tid);
    const uint32_t key = falling_key(allowed ? row.value(tid) : __uint_as_float(0x7FC00000u));
    const RowDraw draw = row_draw(rows, b);
    lds_barrier();
    const unsigned long long candidates = __ballot(is_candidate(key));
    if ((tid & 63) == 0 && candidates) atomicAdd(&s_n, __popcll(candidates));
    if (key == kKeyNegInf) atomicMin(&s_neg_inf, tid);
    lds_barrier();
    const int n = s_n;
    if (n == 0) {
        const bool none = s_neg_inf == vocab;
        if (tid == 0) put_draw(b, none ? -1 : s_neg_inf, none ? -(double)INFINITY : 0.0, none ? 0 : 1, out_tokens, out_logprobs, out_kept);
        return;
    }
    int size = 64;
    while (size < vocab) size *= 2;
    draw_sorted<kBlock>(s, is_candidate(key) ? (unsigned long long)key << 32 | (uint32_t)tid : kNoEntry, size, n, draw, b, out_tokens, out_logprobs, out_kept, tid);
}

// ------------------------------------------------------------------------------- logits of 32 bits

// Logits of 32 bits have too many values to count.  A first pass counts the candidates of 4,096 classes (the first 12 bits of their keys, whose
// order is that of the draw) and finds the maximum, a second one sums the weights of every class and lists the candidates of the first
// classes, as many as the list holds.  A place is found by its class first; then the class's candidates are taken from the list, or, if they are
// not in it, looked at once more, by the next ten bits of their keys and by the last ten.  Weights are summed as whole numbers, in units so
// small that the vocabulary's sum just fits (2^-45 for 128,256 tokens): in whatever order the tokens arrive, the sums are the same.
constexpr int kSampleBlock = 1024, kSampleWaves = kSampleBlock / 64;
constexpr int kClasses = 4096, kDigits = 1024, kListed = 8192;

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
    int likely, listed, n_listed_classes, at, found;
};

// w in units of 2^-bits, to the nearest: the sum with 1.5 * 2^(52 - bits) has them in its last bits.
struct Units {
    double shift;
    unsigned long long zero;
    __device__ explicit Units(int bits) : shift(ldexp(1.5, 52 - bits)), zero(__builtin_bit_cast(unsigned long long, shift)) {}
    __device__ unsigned long long of(double w) const { return __builtin_bit_cast(unsigned long long, w + shift) - zero; }
};

// One pass over a row by a block of kSampleBlock: fn(values, -inf where masked; the first one's id) for eight neighbours at a time,
// by whole waves.
template <class Fn>
__device__ __forceinline__ void each_eight(const Row<LogitsF32> &row, int tid, Fn fn) {
    const int whole = row.vocab >> 3;
    each_group<kSampleBlock, LogitsF32, false>(row, 0, whole, tid, []() { return true; }, [&](int g, const Eight<LogitsF32> *e, const uint32_t *m) {
#pragma unroll
        for (int u = 0; u < kUnroll<LogitsF32>; ++u) {
            if (!__any(m[u] != 0u)) continue;
            float x[8];
            values_of<LogitsF32>(e[u], m[u], nullptr, x);
            fn(x, (g + u * kSampleBlock) * 8);
        }
    });
    if (tid < 64 && (row.vocab & 7)) {
        const int t = whole * 8 + tid;
        const float x[8] = {t < row.vocab && row.allows(t) ? row.value(t) : -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY};
        fn(x, t);
    }
}
// The wanted ones (bit k) of eight into the list, one atomic a wave.
__device__ __forceinline__ void list_some(ClassTables &s, const float *x, uint32_t wanted, int t, int lane) {
    if (!__any(wanted != 0u)) return;
    const int n = __popc(wanted), upto = wave_scan(n);
    int base = 0;
    if (lane == 63) base = atomicAdd(&s.listed, upto);
    int at = from_lane(base, 63) + upto - n;
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if ((wanted >> k) & 1u) {
            s.listed_key[at] = falling_key(x[k]);
            s.listed_id[at++] = t + k;
        }
}
// Sums through the order, in place, kPer entries a thread.
template <int kPer>
__device__ __forceinline__ void sum_through(ClassTables &s, int *count, unsigned long long *weight, int tid) {
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int c[kPer];
    unsigned long long w[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        c[i] = count[tid * kPer + i] + (i ? c[i - 1] : 0);
        w[i] = weight[tid * kPer + i] + (i ? w[i - 1] : 0ull);
    }
    const int count_sum = wave_scan(c[kPer - 1]);
    const unsigned long long weight_sum = wave_scan(w[kPer - 1]);
    if (lane == 63) { s.part_count[wave] = count_sum; s.part[wave] = weight_sum; }
    lds_barrier();
    const int count_parts = wave_scan(lane < kSampleWaves ? s.part_count[lane] : 0);
    const unsigned long long weight_parts = wave_scan(lane < kSampleWaves ? s.part[lane] : 0ull);
    const int count_before = count_sum - c[kPer - 1] + (wave ? from_lane(count_parts, wave - 1) : 0);
    const unsigned long long weight_before = weight_sum - w[kPer - 1] + (wave ? from_lane(weight_parts, wave - 1) : 0ull);
#pragma unroll
    for (int i = 0; i < kPer; ++i) { count[tid * kPer + i] = c[i] + count_before; weight[tid * kPer + i] = w[i] + weight_before; }
    lds_barrier();
}
// The first of such sums (behind c0 and w0) that is what is sought; the last one that has a token where rounding leaves none.  A thread
// looks at its kPer entries if the one before them is not enough and their last one is.
template <int kPer>
__device__ __forceinline__ int first_sought(ClassTables &s, const int *count, const unsigned long long *weight, Sought sought, int c0, unsigned long long w0, int tid) {
    constexpr int kEntries = kPer * kSampleBlock;
    const int all = count[kEntries - 1], from = tid * kPer;
    auto enough = [&](int c, unsigned long long w) { return (sought.tokens ? (double)(c0 + c) : (double)(w0 + w)) > sought.limit || c == all; };
    const int c_before = from ? count[from - 1] : 0, c_last = count[from + kPer - 1];
    if (c_last > c_before && enough(c_last, weight[from + kPer - 1]) && !(from && c_before > 0 && enough(c_before, weight[from - 1]))) {
        int c = c_before;
        for (int i = from; i < from + kPer; ++i) {
            if (count[i] > c && enough(count[i], weight[i])) { s.at = i; break; }
            c = count[i];
        }
    }
    lds_barrier();
    return __builtin_amdgcn_readfirstlane(s.at);
}

__global__ __launch_bounds__(kSampleBlock) void sample_classes_kernel(const uint32_t *__restrict__ logits, const uint32_t *__restrict__ bitmask,
                                                                     int vocab, int64_t row_stride, int n_words, int unit_bits, SampleRows rows,
                                                                     int32_t *__restrict__ out_tokens, float *__restrict__ out_logprobs,
                                                                     int32_t *__restrict__ out_kept) {
    __shared__ __align__(16) ClassTables s;
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.x;
    const Row<LogitsF32> row = {logits + (size_t)b * row_stride, bitmask ? bitmask + (size_t)b * n_words : nullptr, vocab};
    const uint8_t *mask = reinterpret_cast<const uint8_t *>(row.mask);
    const RowDraw draw = row_draw(rows, b);
    const Units units(unit_bits);
    if (tid == 0) { s.best = kKeyNegInf; s.likely = 0; s.listed = 0; s.n_listed_classes = 0; }
    for (int i = tid; i < kClasses; i += kSampleBlock) { s.weight[i] = 0ull; s.upto[i] = 0; }
    lds_barrier();
    // (1) counts and the maximum
    uint32_t best = kKeyNegInf;
    each_eight(row, tid, [&](const float *x, int) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t key = falling_key(x[k]);
            if (is_candidate(key)) {
                best = min(best, key);
                atomicAdd(&s.upto[key >> 20], 1);
            }
        }
    });
    for (int step = 32; step > 0; step /= 2) best = min(best, (uint32_t)__shfl_xor((int)best, step));
    if (lane == 0) atomicMin(&s.best, best);
    lds_barrier();
    best = __builtin_amdgcn_readfirstlane(s.best);
    if (best >= kKeyNegInf) {                  // nothing to draw from
        const int token = find_token<kSampleBlock, 4>(row.logits, mask, vocab, 0, [](uint32_t x) { return x == 0xFF800000u; }, s.part_count, &s.found, tid);
        if (tid == 0) put_draw(b, token, token < 0 ? -(double)INFINITY : 0.0, token < 0 ? 0 : 1, out_tokens, out_logprobs, out_kept);
        return;
    }
    sum_through<kClasses / kSampleBlock>(s, s.upto, s.weight, tid);        // (the weights are all zero yet)
    const int n_all = s.upto[kClasses - 1];
    // (2) weights; the candidates of the first classes, as many as the list holds
    const bool few = n_all <= kSampleBlock;
    int listed_from = 0, listed_to = kClasses; // classes in the list
    if (!few) {
        for (int i = tid; i < kClasses; i += kSampleBlock)
            if (s.upto[i] <= kListed && (i == kClasses - 1 || s.upto[i + 1] > kListed)) s.n_listed_classes = i + 1;
        lds_barrier();
        listed_to = s.n_listed_classes;
    }
    const float top_value = of_falling_key(best);
    const double top = (double)top_value, rate2 = draw.rate * 1.44269504088896340736;
    // the weight as draw_weight has it, in powers of two and with fewer terms (off by 7e-12 of it at most); a maximum of +inf leaves every
    // other weight 0
    const bool infinite = top_value == INFINITY;
    auto weight_of = [=](float x) {
        const double y = fmax(((double)x - top) * rate2, -1100.0), n = rint(y), f = y - n;
        double p = 1.0178086009239696e-07;     // ln(2)^9 / 9!, and so on
        p = fma(p, f, 1.3215486790144305e-06);
        p = fma(p, f, 1.5252733804059838e-05);
        p = fma(p, f, 1.5403530393381606e-04);
        p = fma(p, f, 1.3333558146428441e-03);
        p = fma(p, f, 9.618129107628477e-03);
        p = fma(p, f, 5.5504108664821576e-02);
        p = fma(p, f, 2.402265069591007e-01);
        p = fma(p, f, 6.931471805599453e-01);
        p = fma(p, f, 1.0);
        const double w = ldexp(p, (int)n);
        return infinite ? (x == INFINITY ? 1.0 : 0.0) : w;
    };
    // What goes into the list is weighed there, in 64 bits.  The rest, each a small share of the whole, has weights of 32 bits, which are off by
    // 2^-20 of themselves at most and to either side: sums of thousands of them by 1e-9 of the whole.  Near a border of min-p the
    // 64 bits decide.
    const uint32_t list_end = (uint32_t)listed_to > kKeyNegInf >> 20 ? kKeyNegInf : (uint32_t)listed_to << 20;         // the first key behind the list
    const float rate32 = (float)rate2;
    const double likely_from = draw.min_p > 0.0 ? top + log(draw.min_p) / draw.rate : 0.0;
    const float surely = (float)(likely_from + 1e-6 * fabs(likely_from - top) + 1e-6 * fabs(top)), hardly = (float)(likely_from - 1e-6 * fabs(likely_from - top) - 1e-6 * fabs(top));
    int likely = 0;
    each_eight(row, tid, [&](const float *x, int t) {
        uint32_t first = 0u;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t key = falling_key(x[k]);
            first |= (key - kKeyPosInf < list_end - kKeyPosInf ? 1u : 0u) << k;
            if (key - list_end < kKeyNegInf - list_end) {
                const double w = (double)(infinite ? 0.0f : __builtin_amdgcn_exp2f((x[k] - top_value) * rate32));
                atomicAdd(&s.weight[key >> 20], units.of(w));
            }
        }
        if (draw.min_p > 0.0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t key = falling_key(x[k]);
                if (!(key - list_end < kKeyNegInf - list_end)) continue;
                if (x[k] > surely) ++likely;
                else if (!(x[k] < hardly)) likely += weight_of(x[k]) >= draw.min_p ? 1 : 0;
            }
        }
        list_some(s, x, first, t, lane);
    });
    lds_barrier();
    if (!few) {
        for (int i = tid; i < s.listed; i += kSampleBlock) {
            const uint32_t key = s.listed_key[i];
            const double w = weight_of(of_falling_key(key));
            atomicAdd(&s.weight[key >> 20], units.of(w));
            likely += w >= draw.min_p ? 1 : 0;
        }
    }
    if (few) {                                 // sorted, in place of the weights
        auto &sorted = *reinterpret_cast<Sorted<kSampleBlock> *>(s.weight);
        static_assert(sizeof(Sorted<kSampleBlock>) <= sizeof(s.weight), "the list takes the place of the weights");
        int size = 64;
        while (size < n_all) size *= 2;
        draw_sorted<kSampleBlock>(sorted, tid < n_all ? (unsigned long long)s.listed_key[tid] << 32 | (uint32_t)s.listed_id[tid] : kNoEntry, size, n_all, draw, b, out_tokens,
                                  out_logprobs, out_kept, tid);
        return;
    }
    if (draw.min_p > 0.0) {
        likely = wave_sum(likely);
        if (lane == 0) atomicAdd(&s.likely, likely);
    }
    lds_barrier();
    {                                          // (the counts are summed already)
        const int per = kClasses / kSampleBlock;
        unsigned long long w[per];
#pragma unroll
        for (int i = 0; i < per; ++i) w[i] = s.weight[tid * per + i] + (i ? w[i - 1] : 0ull);
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const unsigned long long sum = wave_scan(w[per - 1]);
        if (lane == 63) s.part[wave] = sum;
        lds_barrier();
        const unsigned long long parts = wave_scan(lane < kSampleWaves ? s.part[lane] : 0ull), before = sum - w[per - 1] + (wave ? from_lane(parts, wave - 1) : 0ull);
#pragma unroll
        for (int i = 0; i < per; ++i) s.weight[tid * per + i] = w[i] + before;
        lds_barrier();
    }
    // (3) one search after the other, as for 16 bits
    int kept = n_all, rank = 0, at_before = 0, at_count = 0;
    double total = (double)s.weight[kClasses - 1], at_weight = 0.0;
    uint32_t at_key = 0u;
    bool in_list = false;
    enum Step { kTopK, kTopP, kMinP, kDraw, kLastKept };
    for (int step = kTopK; step <= kLastKept; ++step) {
        int n = step == kTopK ? draw.top_k : max(s.likely, 1);
        if (step == kTopK && !(draw.top_k > 0 && draw.top_k < kept)) continue;
        if (step == kTopP && !(draw.top_p < 1.0)) continue;
        if (step == kMinP && !(draw.min_p > 0.0 && n < kept)) continue;
        if (step == kLastKept) n = kept;
        const double border = (step == kTopP ? draw.top_p : draw.uniform) * total;
        const Sought sought = step == kTopP ? weight_of_at_least(border) : step == kDraw ? weight_above(border) : first_tokens(n);
        // the class
        lds_barrier();
        const int cls = first_sought<kClasses / kSampleBlock>(s, s.upto, s.weight, sought, 0, 0ull, tid);
        int before = cls ? s.upto[cls - 1] : 0;
        unsigned long long before_weight = cls ? s.weight[cls - 1] : 0ull;
        in_list = cls >= listed_from && cls < listed_to;
        const bool to_list = !in_list && s.upto[cls] - before <= kListed;
        if (to_list) {
            lds_barrier();
            if (tid == 0) s.listed = 0;
            listed_from = cls;
            listed_to = cls + 1;
            in_list = true;
        }
        // the key within it, ten bits at a time
        uint32_t prefix = (uint32_t)cls;
        for (int level = 0; level < 2; ++level) {
            const int shift = level ? 0 : 10;
            lds_barrier();
            s.digit_count[tid] = 0;
            s.digit_weight[tid] = 0ull;
            lds_barrier();
            auto add = [&](uint32_t key) {
                if (key >> (shift + 10) != prefix) return;
                atomicAdd(&s.digit_count[(key >> shift) & 1023u], 1);
                atomicAdd(&s.digit_weight[(key >> shift) & 1023u], units.of(weight_of(of_falling_key(key))));
            };
            if (!in_list || (to_list && level == 0)) {
                each_eight(row, tid, [&](const float *x, int t) {
                    uint32_t wanted = 0u;
#pragma unroll
                    for (int k = 0; k < 8; ++k) wanted |= (falling_key(x[k]) >> 20 == (uint32_t)cls && is_candidate(falling_key(x[k])) ? 1u : 0u) << k;
                    if (in_list) list_some(s, x, wanted, t, lane);
                    else
                        for (uint32_t left = wanted; left; left &= left - 1u) {
                            const int k = __ffs(left) - 1;
                            add(falling_key(k == 0 ? x[0] : k == 1 ? x[1] : k == 2 ? x[2] : k == 3 ? x[3] : k == 4 ? x[4] : k == 5 ? x[5] : k == 6 ? x[6] : x[7]));
                        }
                });
                lds_barrier();
            }
            if (in_list) {
                for (int i = tid; i < s.listed; i += kSampleBlock) add(s.listed_key[i]);
                lds_barrier();
            }
            sum_through<1>(s, s.digit_count, s.digit_weight, tid);
            const int digit = first_sought<kDigits / kSampleBlock>(s, s.digit_count, s.digit_weight, sought, before, before_weight, tid);
            const int c = digit ? s.digit_count[digit - 1] : 0;
            at_count = s.digit_count[digit] - c;
            before += c;
            before_weight += digit ? s.digit_weight[digit - 1] : 0ull;
            prefix = prefix << 10 | (uint32_t)digit;
        }
        at_key = prefix;
        at_before = before;
        at_weight = weight_of(of_falling_key(at_key));
        const unsigned long long w = units.of(at_weight);
        if (step == kTopP) {                   // tokens of the value with less than the border before them
            const double r = ceil((border - (double)before_weight) / (double)w);
            n = before + (r >= at_count ? at_count : r >= 1.0 ? (int)r : 1);
        }
        if (step < kDraw) {
            if (n < kept) { kept = n; total = (double)(before_weight + w * (unsigned long long)(n - before)); }
            continue;
        }
        const double r = floor((border - (double)before_weight) / (double)w);
        rank = step == kLastKept ? kept - 1 - before : r >= at_count ? at_count - 1 : r >= 1.0 ? (int)r : 0;
        if (step == kLastKept || at_before + rank < kept) break;           // (else rounding, or a number that is not below 1: the last of those kept)
    }
    // (4) the id
    int token;
    if (in_list && at_count == 1) {
        for (int i = tid; i < s.listed; i += kSampleBlock)
            if (s.listed_key[i] == at_key) s.found = s.listed_id[i];
        lds_barrier();
        token = s.found;
    } else {
        const uint32_t key = at_key;
        token = find_token<kSampleBlock, 4>(row.logits, mask, vocab, rank, [=](uint32_t x) { return falling_key(__uint_as_float(x)) == key; }, s.part_count, &s.found, tid);
    }
    if (tid == 0) put_draw(b, token, log(at_weight * ldexp(1.0, unit_bits) / total), kept, out_tokens, out_logprobs, out_kept);
}

template <class F>
void launch_sorted(const void *logits, const uint32_t *bitmask, int batch, int vocab, int64_t row_stride, int n_words, const SampleRows &rows,
                   int32_t *out_tokens, float *out_logprobs, int32_t *out_kept, hipStream_t stream) {
    auto go = [&](auto kernel, int block) {
        hipLaunchKernelGGL(kernel, dim3(batch), dim3(block), 0, stream, static_cast<const typename F::Stored *>(logits), bitmask, vocab, row_stride, n_words, rows,
                           out_tokens, out_logprobs, out_kept);
    };
    if (vocab <= 256) go(sample_sorted_kernel<256, F>, 256);
    else go(sample_sorted_kernel<kSampleBlock, F>, kSampleBlock);
}

}  // namespace

hipError_t launch_masked_sample(const void *logits, LogitType type, const uint32_t *bitmask, int batch, int vocab, int64_t row_stride,
                                const SampleRows &rows, int32_t *out_tokens, float *out_logprobs, int32_t *out_kept, hipStream_t stream) {
    if (batch == 0) return hipSuccess;
    const int n_words = (vocab + 31) / 32;
    auto launch = [&](auto fn, auto... first) { fn(first..., bitmask, batch, vocab, row_stride, n_words, rows, out_tokens, out_logprobs, out_kept, stream); };
    if (vocab <= kSampleBlock) {
        if (type == kLogitBf16) launch(launch_sorted<LogitsBf16>, logits);
        else if (type == kLogitF16) launch(launch_sorted<LogitsF16>, logits);
        else launch(launch_sorted<LogitsF32>, logits);
    } else if (type == kLogitBf16) {
        launch(launch_counts<Bf16>, static_cast<const uint16_t *>(logits));
    } else if (type == kLogitF16) {
        launch(launch_counts<F16>, static_cast<const uint16_t *>(logits));
    } else {
        int bits = 52;                          // the vocabulary's sum of weights stays below 2^63, and a weight's units below 2^51
        while (bits > 30 && ((int64_t)1 << (62 - bits)) < vocab) --bits;
        if (bits > 50) bits = 50;
        hipLaunchKernelGGL(sample_classes_kernel, dim3(batch), dim3(kSampleBlock), 0, stream, static_cast<const uint32_t *>(logits), bitmask, vocab, row_stride,
                           n_words, bits, rows, out_tokens, out_logprobs, out_kept);
    }
    return hipGetLastError();
}

}  // namespace pre3
