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
// e^x for x <= 0 in 64 bits: x = n ln 2 + r with |r| <= ln 2 / 2 (Cody and Waite's reduction) and the exponential series of r up to r^12 / 12! (the next term is
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
// block; every thread gets it.  s_part: a word per wave.  s_found: a word that nothing else uses, since it is written before the first
// barrier, when other waves may still be looking at what the caller has in LDS.
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

// Up to a thousand candidates are sorted, key above id, and everything is a place among them.  A wave sorts its 64 by a bitonic network with
// moves between lanes; runs are merged two by two, every entry finding its place in the other run by bisection: one barrier
// for a doubling.  (With the whole network, through LDS beyond a wave: 4 x 513 12.5 us a launch, now 10.8.)
template <int kBlock>
struct Sorted {
    unsigned long long entry[kBlock];
    union {
        unsigned long long merged[kBlock];
        double upto[kBlock];                   // weights summed, the place included
    };
    double part[kBlock / 64];
    int likely;
};
constexpr unsigned long long kNoEntry = ~0ull;
template <int kBit>
__device__ __forceinline__ uint32_t lane_across(uint32_t x, int lane) {                 // lane ^ kBit's
    if constexpr (kBit == 1) return lane_move<0xB1, 0xF>(x);
    else if constexpr (kBit == 2) return lane_move<0x4E, 0xF>(x);
    else if constexpr (kBit == 4) return lane_move<0x1B, 0xF>(lane_move<0x141, 0xF>(x));     // (7 and 3)
    else if constexpr (kBit == 8) return lane_move<0x128, 0xF>(x);
    else {
        const auto two = [&]() {
            if constexpr (kBit == 16) return __builtin_amdgcn_permlane16_swap(x, x, false, false);
            else return __builtin_amdgcn_permlane32_swap(x, x, false, false);
        }();
        return lane & kBit ? two[0] : two[1];
    }
}
template <int kRun, int kBit>
__device__ __forceinline__ void bitonic(unsigned long long &mine, int lane) {
    const unsigned long long other = (unsigned long long)lane_across<kBit>((uint32_t)(mine >> 32), lane) << 32 | lane_across<kBit>((uint32_t)mine, lane);
    const bool smaller = ((lane & kBit) == 0) == ((lane & kRun) == 0);       // this lane keeps the smaller of the two
    mine = (other < mine) == smaller ? other : mine;
    if constexpr (kBit > 1) bitonic<kRun, kBit / 2>(mine, lane);
}
__device__ __forceinline__ unsigned long long sorted_in_wave(unsigned long long mine, int lane) {
    bitonic<2, 1>(mine, lane);
    bitonic<4, 2>(mine, lane);
    bitonic<8, 4>(mine, lane);
    bitonic<16, 8>(mine, lane);
    bitonic<32, 16>(mine, lane);
    bitonic<64, 32>(mine, lane);
    return mine;
}
// Sorts s.entry; each thread's entry of the first `size`, a power of two from 64 on, before and after.
template <int kBlock>
__device__ __forceinline__ unsigned long long sorted_entry(Sorted<kBlock> &s, unsigned long long mine, int size, int tid) {
    unsigned long long *from = s.entry, *to = s.merged;
    if (tid < size) mine = sorted_in_wave(mine, tid & 63);
    lds_barrier();
    from[tid] = mine;
    lds_barrier();
    for (int run = 64; run < size; run *= 2) {
        const int pair = tid & ~(2 * run - 1), at = tid & (run - 1);
        const bool second = (tid & run) != 0;
        const unsigned long long *other = from + pair + (second ? 0 : run);
        int lo = 0;                            // of the other run's entries, those before this one (equal ones, which are no candidates: the first run's)
        if (tid < size) {
            for (int step = run / 2; step > 0; step /= 2) {
                const unsigned long long x = other[lo + step - 1];
                if (second ? x <= mine : x < mine) lo += step;
            }
            const unsigned long long x = other[lo];
            if (second ? x <= mine : x < mine) ++lo;
            to[pair + at + lo] = mine;
        }
        lds_barrier();
        if (tid < size) mine = to[tid];
        unsigned long long *swap = from;
        from = to;
        to = swap;
    }
    if (from != s.entry) {
        s.entry[tid] = mine;
        lds_barrier();
    }
    return mine;
}
// The draw from n >= 1 candidates, each thread's entry a key above an id or kNoEntry, the first `size` (a power of two) threads' ones all there are.
template <int kBlock>
__device__ __forceinline__ void draw_sorted(Sorted<kBlock> &s, unsigned long long mine, int size, int n, const RowDraw &draw, int b, int32_t *out_tokens, float *out_logprobs,
                                            int32_t *out_kept, int tid) {
    if (tid == 0) s.likely = 0;
    mine = sorted_entry<kBlock>(s, mine, size, tid);
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
    mine = sorted_in_wave(mine, lane);
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
    static constexpr bool kByOctave = false;               // (a segment is two octaves)
    __device__ static double value(uint32_t h) { return (double)__uint_as_float(h << 16); }
};
struct F16 {
    static constexpr uint32_t kInf = 0x7C00u;
    static constexpr bool kByOctave = true;
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

// Four segments of one octave at once, 4 q .. 4 q + 3, without infinities and without the row's maximum: sixteen neighbouring values a lane, whose
// weights are the first one's times powers of a factor.  (f16 spreads a row over some 150 segments: 96 x 100,003 one by one 25.4 us a launch, so 21.9.)
template <class F, bool kNegative>
__device__ __forceinline__ int sum_octave(CountTables &s, int q, double top, double rate, int lane) {
    constexpr int kOctave = 4 * kSegmentWords, kSide = kWords / kOctave, kPer = kOctave / 64;
    const uint32_t low = (uint32_t)(kNegative ? q - kSide : kSide - 1 - q) * kOctave + (uint32_t)(kNegative ? lane * kPer : kOctave - kPer - lane * kPer);
    const double value = F::value(kNegative ? low | 0x8000u : low + kPer - 1), next = F::value(kNegative ? low | 0x8001u : low + kPer - 2);
    const double factor = exp_of_negative((next - value) * rate), first = exp_of_negative((value - top) * rate);
    int tokens = 0;
    double weight = 0.0;
#pragma unroll
    for (int j = kPer / 4 - 1; j >= 0; --j) {              // from the last value in the order to the first
        const uint4 x = *reinterpret_cast<const uint4 *>(s.count + low + (kNegative ? 4 * j : kPer - 4 - 4 * j));
        const uint32_t c[4] = {kNegative ? x.w >> 16 : x.x & 0xFFFFu, kNegative ? x.z >> 16 : x.y & 0xFFFFu,
                               kNegative ? x.y >> 16 : x.z & 0xFFFFu, kNegative ? x.x >> 16 : x.w & 0xFFFFu};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            tokens += (int)c[i];
            weight = fma(weight, factor, (double)c[i]);
        }
    }
    weight *= first;
    // sums over the sixteen lanes of a segment, in its last one
    tokens += lane_move_of<0x111, 0xF>(tokens); weight += lane_move_of<0x111, 0xF>(weight);
    tokens += lane_move_of<0x112, 0xF>(tokens); weight += lane_move_of<0x112, 0xF>(weight);
    tokens += lane_move_of<0x114, 0xF>(tokens); weight += lane_move_of<0x114, 0xF>(weight);
    tokens += lane_move_of<0x118, 0xF>(tokens); weight += lane_move_of<0x118, 0xF>(weight);
    const bool last = (lane & 15) == 15;
    if (last) { s.tokens[q * 4 + (lane >> 4)] = tokens; s.weight[q * 4 + (lane >> 4)] = weight; }
    return last ? tokens : 0;
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
        if (step == kDraw && !(draw.uniform < 1.0)) continue;          // (the last token kept, also where its weight is zero)
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

// One block a row of more than kSampleBlock tokens, kG groups of eight a thread; a row of more than a block's kG * 8,192 tokens (kMany) goes through in chunks and is
// read again for the token's id.
// 256 x 128,256 with mixed filters: 24 us a launch, 2.8 TB/s.  The stream ends at 13 us (the first groups and the mask are there at 3.4, two
// tokens cost ten instructions and two LDS adds); what follows is the latency of a block's steps: the segments with tokens until
// 14.6, their weights 16.9, the draw by one wave 20.8, the id 23.2.  One row alone takes 17 us: its unit counts until 11.
template <class F, int kG, bool kMany>
__global__ __launch_bounds__(kCountBlock) void sample_counts_kernel(const uint16_t *__restrict__ logits, const uint32_t *__restrict__ bitmask,
                                                                    int vocab, int64_t row_stride, int n_words, SampleRows rows,
                                                                    int32_t *__restrict__ out_tokens, float *__restrict__ out_logprobs,
                                                                    int32_t *__restrict__ out_kept) {
    // (groups asked for before the mask is there: with eight, rows of few tokens fetch what they do not need, 512 x 152,064 schema 58.0 us, 56.0 with three)
    constexpr int kAhead = kG < 3 ? kG : 3, kLook = kHalf / kCountWaves;                  // groups in flight; looks at the words of a segment a wave
    constexpr int kKept = kG < 12 ? kG : 12;              // groups that stay in registers through the draw (all 20: 45 registers spilled)
    __shared__ __align__(16) CountTables s;
    struct Group { uint4 x; uint32_t allowed; int at; };
    __shared__ Group s_rest;
    __shared__ uint2 s_ones[16];                          // four mask bits -> 1 or 0 in the halves of two registers
    __shared__ uint16_t s_busy[kSegments];                // segments that have tokens
    __shared__ uint8_t s_octave[kSegments / 4];           // whether one of four has
    __shared__ int s_first, s_likely, s_seen, s_n_busy, s_listed, s_equal, s_token_found, s_part[kCountWaves], s_id[kCountBlock];
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
        for (int u = 0; u < kG; ++u) m[u] = mask ? mask[min((uint32_t)(first + u * kCountBlock), (uint32_t)whole - 1u)] : 0xFFu;      // (unsigned: no sign to extend, 44.2 -> 43.1 us on 512 x 152,064 schema)
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
#pragma unroll
        for (int u = from; u < to; ++u) load(chunk, u);
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
    // (1) counts; a row of which the mask allows at most 64 tokens is one wave's instead (256 x 128,256 with 30 allowed tokens: 17.0 us
    // by counts, 8.3 by a wave.  Rows of up to 1,024, sorted by the block, lost: 900 allowed tokens 21.6 by counts, 26.5 sorted)
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
    if (F::kByOctave && tid < kSegments / 4) s_octave[tid] = 0;
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
            if (F::kByOctave) s_octave[seg >> 2] = 1;
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
        const int token = find_pattern(row, mask, vocab, 0, F::kInf | 0x8000u, 0xFFFFu, s_part, &s_token_found);
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
    auto sum_segment = [&](int seg) {
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
    };
    if (F::kByOctave && n_heavy == 0) {
        const double limit = draw.min_p > 0.0 ? top.value + log(draw.min_p) / draw.rate : 0.0, margin = 1e-6 * (fabs(limit) + 1.0);
        for (int q = wave; q < kSegments / 4; q += kCountWaves) {
            if (!__builtin_amdgcn_readfirstlane(s_octave[q])) continue;
            const bool negative = q >= kSegments / 8;
            const double ends[2] = {F::value(word_at(4 * q, 0) | (negative ? 0x8000u : 0u)), F::value(word_at(4 * q + 3, kSegmentWords - 1) | (negative ? 0x8000u : 0u))};
            const bool above = draw.min_p > 0.0 && ends[1] > limit + margin, below = !(draw.min_p > 0.0) || ends[0] < limit - margin;
            if (q == 0 || q == top.seg >> 2 || !(above || below)) {              // (0: +inf and the NaNs)
                for (int i = 0; i < 4; ++i) sum_segment(4 * q + i);
            } else {
                const int tokens = negative ? sum_octave<F, true>(s, q, top.value, draw.rate, lane) : sum_octave<F, false>(s, q, top.value, draw.rate, lane);
                if (above) likely += tokens;
            }
        }
    } else {
        for (int i = wave; i < n_busy; i += kCountWaves) sum_segment(__builtin_amdgcn_readfirstlane(s_busy[i]));
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
        const int token = find_pattern(row, mask, vocab, rank, pattern, care, s_part, &s_token_found);
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

// Vocabularies of up to kBlock tokens.  Bound by the latency of one block (4 x 513: 10.4 us a launch).
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

// Logits of 32 bits have too many values to count.  A first pass finds the largest and the smallest candidate.  The second one gives every
// candidate a bin by its distance d to the largest, bin = round(d * scale), which keeps the order of the draw: 4,096 bins over the row's
// range, or over 64 octaves of weight if it spans more (what lies farther weighs nothing, 2^-45 of the row at most, and is counted only).
// Within a bin a weight is that of the bin's middle times 1 + e, |e| <= 0.0055, so that one 64-bit atomic adds a token and its e:
// the count in the upper 20 bits, e in units of 2^-31 in the lower 44.  Whole numbers: in whatever order the tokens arrive, the sums are
// the same, and a bin's weight is right to 2^-32 of itself.  Sums over the bins say in which bin each border lies, before any of the places
// is known exactly; a third pass lists the candidates of these few bins, which are sorted once, and every place is one in that list.
// A bin that the list has no room for (values that hundreds of tokens share) is looked at digit by digit of its keys.
// 128 x 128,256, top-p: 52.6 us a launch.  Bound by instructions (one a token is 0.83 us a row: a wave's takes four cycles) and by the LDS
// atomics: 9 to 11 us for the first pass, 17 for the second, 9 to 12 for the third.  Counting classes of the keys' first bits and adding weights to
// them with atomics, which meet on few addresses, took 104.
constexpr int kSampleBlock = 1024, kSampleWaves = kSampleBlock / 64;
constexpr int kBins = 4096, kDigits = 2048;
constexpr double kMostOctaves = 64.0, kBinEnd = kBins - 1.0;                // bins of distances below kBinEnd
constexpr int kCountShift = 44, kPartBits = 31;
constexpr float kLowest = -3.40282346638528859812e+38f;   // the smallest candidate there can be
constexpr int kRest = -1;                                 // the "bin" of the candidates beyond the last one

// The first of `n` <= 4,096 places from which on it holds, by a wave (every one for itself, without barriers); n: none.
template <class Holds>
__device__ __forceinline__ int first_place(int n, int lane, Holds holds) {
    const int per = (n + 63) / 64;
    const int last = min((lane + 1) * per, n) - 1;
    const unsigned long long coarse = __ballot(holds(last));
    if (coarse == 0ull) return n;
    const int from = (__ffsll(coarse) - 1) * per, at = from + lane;
    const unsigned long long fine = __ballot(lane < per && at < n && holds(min(at, n - 1)));
    return __builtin_amdgcn_readfirstlane(fine ? from + __ffsll(fine) - 1 : min(from + per, n) - 1);
}
// Distances into bins.
struct Binning {
    double scale, origin;                     // bins a unit of the logits; the largest logit times that
    double octave;                            // octaves of the weight a bin
    double c1, c2, c3;                        // e of a place f beside a bin's middle, in units: f (c1 + f (c2 + f c3))
    static constexpr double kRound = 6755399441055744.0;                    // 1.5 * 2^52: a sum with it ends at the ones
    __device__ void set(double top, double smallest, double rate) {
        const double rate2 = rate * 1.44269504088896340736;
        double octaves = (top - smallest) * rate2;
        if (!(octaves < kMostOctaves) || octaves < 1e-200) octaves = kMostOctaves;
        // (29 bits of it: its products with the 24 of a logit are exact)
        scale = __builtin_bit_cast(double, __builtin_bit_cast(unsigned long long, rate2 * (kBinEnd - 5.0) / octaves) & ~0xFFFFFFull);
        octave = rate2 / scale;               // (scale is zero only where the rate is)
        if (!(scale > 0.0)) octave = 0.0;
        origin = top * scale;
        const double l = 0.693147180559945309417 * octave, unit = (double)(1ull << kPartBits);
        c1 = -l * unit; c2 = l * l * (0.5 * unit); c3 = -l * l * l * (unit / 6);
    }
    // In bins; infinite, or a NaN, as x is.
    __device__ double place(float x) const { return fma((double)x, -scale, origin); }
    __device__ static int bin_of(double place) { return (int)(uint32_t)__builtin_bit_cast(unsigned long long, place + kRound); }
    // what a token adds to its bin
    __device__ unsigned long long entry(double place, double rounded) const {
        const double f = place - (rounded - kRound), e = fma(f, fma(f, fma(f, c3, c2), c1), kRound);
        const unsigned long long bits = __builtin_bit_cast(unsigned long long, e);
        constexpr uint32_t kOne = 0x43380000u - (1u << (kCountShift - 32));  // (the upper half of kRound, less a token)
        return (unsigned long long)((uint32_t)(bits >> 32) - kOne) << 32 | (uint32_t)bits;
    }
    __device__ double weight(int bin) const { return exp_of_negative(bin * -0.693147180559945309417 * octave); }
};
// What the searches of a row go by.  A largest logit of +inf has the first bin to itself, and the others weigh nothing.
struct RowBins {
    RowDraw draw;
    Binning binning;
    float top;
    int n_all, likely;                        // likely: the tokens with a weight of min_p and more, -1: not known yet
    bool infinite;
};
struct BinTables {
    unsigned long long weight[kBins];         // first counts and parts, then (a double) the weight through the order, the bin included
    int tokens[kBins];                        // through the order, the bin included
    uint8_t listed[kBins];                    // whether the list has the bin
    int start[kBins];                         // of the listed bins: place of the first token in the list
    unsigned long long digit_weight[kDigits]; // as for the bins
    int digit_tokens[kDigits];
    Sorted<kSampleBlock> sorted;
    double part[kSampleWaves];
    int part_tokens[kSampleWaves], n_listed, likely, likely_from, likely_to, token_found, n_ranges, done;
    float largest[kSampleWaves], smallest[kSampleWaves], middle[4], half[4];     // ranges of logits, and a little more: those in the listed bins
    RowBins row;

    __device__ double weight_through(int bin) const { return __builtin_bit_cast(double, weight[bin]); }
    __device__ double weight_before(int bin) const { return bin ? weight_through(bin - 1) : 0.0; }
    __device__ int tokens_before(int bin) const { return bin ? tokens[bin - 1] : 0; }
    __device__ int in_bins() const { return tokens[kBins - 1]; }
    // by a wave, every one for itself
    __device__ int bin_with(int n, int lane) const { return min(first_place(kBins, lane, [&](int i) { return tokens[i] >= n; }), kBins - 1); }
    __device__ int bin_reaching(const Sought &sought, int lane) const {
        const int bin = min(first_place(kBins, lane, [&](int i) { return weight_through(i) > sought.limit; }), kBins - 1);
        return tokens[bin] > tokens_before(bin) ? bin : bin_with(max(tokens[bin], 1), lane);  // (rounding: the last bin before it that has tokens)
    }
};

// One pass over a row by a block of kSampleBlock: fn(values, NaN where masked; the first one's id; the mask byte) for eight neighbours at a
// time, by whole waves.  kRaw: values as they are, masked or not.
template <bool kRaw = false, class Fn>
__device__ __forceinline__ void each_eight(const Row<LogitsF32> &row, int tid, Fn fn) {
    const int whole = row.vocab >> 3;
    each_group<kSampleBlock, LogitsF32, false>(row, 0, whole, tid, []() { return true; }, [&](int g, const Eight<LogitsF32> *e, const uint32_t *m) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (!__any(m[u] != 0u)) continue;
            const uint32_t w[8] = {e[u].v[0].x, e[u].v[0].y, e[u].v[0].z, e[u].v[0].w, e[u].v[1].x, e[u].v[1].y, e[u].v[1].z, e[u].v[1].w};
            const int masked = (int)~m[u];
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(kRaw ? w[i] : w[i] | (uint32_t)__builtin_amdgcn_sbfe(masked, i, 1));
            fn(x, (g + u * kSampleBlock) * 8, m[u]);
        }
    });
    if (tid < 64 && (row.vocab & 7)) {
        const int t = whole * 8 + tid;
        const float none = __uint_as_float(0x7FC00000u);
        const float x[8] = {t < row.vocab && row.allows(t) ? row.value(t) : none, none, none, none, none, none, none, none};
        fn(x, t, 1u);
    }
}
// Sums through the order, in place, kPer entries a thread, of which the first has tokens of the weight `unit`, each further one of `ratio` times that.
template <int kPer>
__device__ __forceinline__ void sum_through(BinTables &s, unsigned long long *weight, int *tokens, double unit, double ratio, int tid) {
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int c[kPer];
    double w[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const unsigned long long x = weight[tid * kPer + i];
        const int n = (int)((x + (1ull << (kCountShift - 1))) >> kCountShift);
        const long long part = (long long)(x - ((unsigned long long)n << kCountShift));
        c[i] = n + (i ? c[i - 1] : 0);
        w[i] = unit * fma((double)part, 1.0 / (1ull << kPartBits), (double)n) + (i ? w[i - 1] : 0.0);
        unit *= ratio;
    }
    const int count_sum = wave_scan(c[kPer - 1]);
    const double weight_sum = wave_scan(w[kPer - 1]);
    if (lane == 63) { s.part_tokens[wave] = count_sum; s.part[wave] = weight_sum; }
    lds_barrier();
    const int count_parts = wave_scan(lane < kSampleWaves ? s.part_tokens[lane] : 0);
    const double weight_parts = wave_scan(lane < kSampleWaves ? s.part[lane] : 0.0);
    const int count_before = count_sum - c[kPer - 1] + (wave ? from_lane(count_parts, wave - 1) : 0);
    const double weight_before = (wave ? from_lane(weight_parts, wave - 1) : 0.0) + (weight_sum - w[kPer - 1]);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        tokens[tid * kPer + i] = c[i] + count_before;
        weight[tid * kPer + i] = __builtin_bit_cast(unsigned long long, w[i] + weight_before);
    }
    lds_barrier();
}

// A value of the order: the tokens before it with their weight, its number of tokens.
struct ValuePlace { uint32_t key; int before, count; double ahead; };
// The value in a bin that is not in the list, by the whole block: ten and twice eleven bits of the key at a time.
__device__ __forceinline__ ValuePlace place_by_digits(BinTables &s, const RowBins &r, const Row<LogitsF32> &row, int bin, bool by_tokens, int n, double limit, int tid) {
    const int lane = tid & 63;
    const bool rest = bin == kRest;
    ValuePlace p = {0u, rest ? s.in_bins() : s.tokens_before(bin), 0, rest ? s.weight_through(kBins - 1) : s.weight_before(bin)};
    const double unit = rest ? 0.0 : r.binning.weight(bin);
    int shift = 22;
    for (int level = 0; level < 3; ++level, shift -= 11) {
        lds_barrier();
        for (int i = tid; i < kDigits; i += kSampleBlock) s.digit_weight[i] = 0ull;
        lds_barrier();
        each_eight(row, tid, [&](const float *x, int, uint32_t) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (!(x[k] >= kLowest)) continue;
                const uint32_t digits = falling_key(x[k]) >> shift;
                if (level && digits >> 11 != p.key) continue;
                const double place = r.binning.place(x[k]);
                const bool inside = r.infinite ? x[k] == INFINITY : place < kBinEnd;
                if (rest ? inside : !inside || Binning::bin_of(place) != bin) continue;
                atomicAdd(&s.digit_weight[digits & (level ? 2047u : 1023u)], rest ? 1ull << kCountShift : r.binning.entry(place, place + Binning::kRound));
            }
        });
        lds_barrier();
        sum_through<kDigits / kSampleBlock>(s, s.digit_weight, s.digit_tokens, unit, 1.0, tid);
        auto weight_of = [&](int i) { return __builtin_bit_cast(double, s.digit_weight[i]); };
        int digit = first_place(kDigits, lane, [&](int i) { return by_tokens ? p.before + s.digit_tokens[i] >= n : p.ahead + weight_of(i) > limit; });
        digit = min(digit, kDigits - 1);
        if (s.digit_tokens[digit] == (digit ? s.digit_tokens[digit - 1] : 0)) {      // (rounding, as for the bins)
            const int at = max(s.digit_tokens[digit], 1);
            digit = first_place(kDigits, lane, [&](int i) { return s.digit_tokens[i] >= at; });
        }
        const int c = digit ? s.digit_tokens[digit - 1] : 0;
        p.count = s.digit_tokens[digit] - c;
        p.before += c;
        p.ahead += digit ? weight_of(digit - 1) : 0.0;
        p.key = p.key << (level ? 11 : 0) | (uint32_t)digit;
    }
    return p;
}

// What is kept, and the draw: one search after the other, as for 16 bits.  By wave 0, as long as the list has every place (else `found` is
// false), or by the whole block.  (With all waves at it, and at the borders: 128 x 128,256 top-p 60.9 us, so 52.4.)
struct DrawnToken { bool found, by_id; int kept, token, rank; uint32_t key; double logprob; };
template <bool kByBlock>
__device__ __forceinline__ DrawnToken draw_from_bins(BinTables &s, const RowBins &r, const Row<LogitsF32> &row, int tid) {
    const int lane = tid & 63, in_bins = s.in_bins();
    DrawnToken d = {true, false, r.n_all, -1, 0, 0u, 0.0};
    double total = s.weight_through(kBins - 1);
    enum Step { kTopK, kTopP, kMinP, kDraw, kLastKept };
    for (int step = kTopK; step <= kLastKept; ++step) {
        int n = step == kTopK ? r.draw.top_k : max(r.likely, 1);
        if (step == kTopK && !(r.draw.top_k > 0 && r.draw.top_k < d.kept)) continue;
        if (step == kTopP && !(r.draw.top_p < 1.0)) continue;
        if (step == kMinP && !(r.draw.min_p > 0.0 && n < d.kept)) continue;
        if (step == kDraw && !(r.draw.uniform < 1.0)) continue;
        if (step == kLastKept) n = d.kept;
        const bool by_tokens = step != kTopP && step != kDraw;
        const double border = (step == kTopP ? r.draw.top_p : r.draw.uniform) * total;
        const Sought sought = step == kTopP ? weight_of_at_least(border) : step == kDraw ? weight_above(border) : first_tokens(n);
        const int bin = !by_tokens ? s.bin_reaching(sought, lane) : n <= in_bins ? s.bin_with(n, lane) : kRest;
        if (step == kTopK || step == kMinP) {  // whole bins need no place
            if (bin == kRest || s.tokens[bin] == n) {
                total = s.weight_through(bin == kRest ? kBins - 1 : bin);
                d.kept = n;
                continue;
            }
        }
        ValuePlace p;
        d.by_id = bin != kRest && s.listed[bin] != 0;
        if (d.by_id) {
            const int before = s.tokens_before(bin), from = s.start[bin], size = s.tokens[bin] - before;
            const double ahead = s.weight_before(bin), offset = ahead - (from ? s.sorted.upto[from - 1] : 0.0);
            const int i = by_tokens ? n - before - 1
                                    : min(first_place(size, lane, [&](int k) { return offset + s.sorted.upto[from + k] > sought.limit; }), size - 1);
            const unsigned long long entry = s.sorted.entry[from + i];
            p = {(uint32_t)(entry >> 32), before + i, 1, i ? offset + s.sorted.upto[from + i - 1] : ahead};
            d.token = (int)(uint32_t)entry;
        } else if (r.infinite && bin == 0) {
            p = {kKeyPosInf, 0, in_bins, 0.0};
        } else if (kByBlock) {
            p = place_by_digits(s, r, row, bin, by_tokens, n, sought.limit, tid);
        } else {
            d.found = false;
            return d;
        }
        const double weight = draw_weight((double)of_falling_key(p.key), (double)r.top, r.draw.rate);
        if (step == kTopP) {                   // tokens of the value with less than the border before them
            const double q = ceil((border - p.ahead) / weight);
            n = p.before + (q >= p.count ? p.count : q >= 1.0 ? (int)q : 1);
        }
        if (step < kDraw) {
            if (n < d.kept) { d.kept = n; total = p.ahead + weight * (n - p.before); }
            continue;
        }
        const double q = floor((border - p.ahead) / weight);
        d.rank = step == kLastKept ? d.kept - 1 - p.before : q >= p.count ? p.count - 1 : q >= 1.0 ? (int)q : 0;
        if (step == kDraw && p.before + d.rank >= d.kept) continue;        // (rounding: the last of those kept)
        d.key = p.key;
        d.logprob = log(weight / total);
        break;
    }
    return d;
}
// The draw of a row whose list lacks a place, from what s.row says.  By the block; a call of its own: such rows are rare.
__device__ __noinline__ void draw_by_block(BinTables &s, const uint32_t *logits, const uint32_t *bitmask, int vocab, int b, int32_t *out_tokens, float *out_logprobs,
                                           int32_t *out_kept) {
    const int tid = threadIdx.x;
    const Row<LogitsF32> row = {logits, bitmask, vocab};
    const uint8_t *mask = reinterpret_cast<const uint8_t *>(bitmask);
    RowBins r = s.row;
    if (r.draw.min_p > 0.0 && r.likely < 0) {
        lds_barrier();
        if (tid == 0) s.likely = 0;
        lds_barrier();
        each_eight(row, tid, [&](const float *x, int, uint32_t) {
            int n = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) n += x[k] >= kLowest && draw_weight((double)x[k], (double)r.top, r.draw.rate) >= r.draw.min_p ? 1 : 0;
            if (n) atomicAdd(&s.likely, n);
        });
        lds_barrier();
        r.likely = s.likely;
    }
    DrawnToken d = draw_from_bins<true>(s, r, row, tid);
    if (!d.by_id) {                            // the token by its place among the equal ones
        const uint32_t key = d.key;
        d.token = find_token<kSampleBlock, 4>(logits, mask, vocab, d.rank, [=](uint32_t x) { return falling_key(__uint_as_float(x)) == key; }, s.part_tokens, &s.token_found, tid);
    }
    if (tid == 0) put_draw(b, d.token, d.logprob, d.kept, out_tokens, out_logprobs, out_kept);
}
// The first allowed -inf of a row without candidates, or none.  A call of its own.
__device__ __noinline__ int first_neg_inf(BinTables &s, const uint32_t *logits, const uint32_t *bitmask, int vocab) {
    return find_token<kSampleBlock, 4>(logits, reinterpret_cast<const uint8_t *>(bitmask), vocab, 0, [](uint32_t x) { return x == 0xFF800000u; }, s.part_tokens, &s.token_found,
                                       threadIdx.x);
}

__global__ __launch_bounds__(kSampleBlock) void sample_bins_kernel(const uint32_t *__restrict__ logits, const uint32_t *__restrict__ bitmask,
                                                                  int vocab, int64_t row_stride, int n_words, SampleRows rows,
                                                                  int32_t *__restrict__ out_tokens, float *__restrict__ out_logprobs,
                                                                  int32_t *__restrict__ out_kept) {
    __shared__ __align__(16) BinTables s;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
    const Row<LogitsF32> row = {logits + (size_t)b * row_stride, bitmask ? bitmask + (size_t)b * n_words : nullptr, vocab};
    RowBins r;
    r.draw = row_draw(rows, b);
    if (tid == 0) { s.likely = 0; s.n_listed = 0; }
    for (int i = tid; i < kBins; i += kSampleBlock) { s.weight[i] = 0ull; s.listed[i] = 0; }
    // (1) the candidates' number, the largest and the smallest
    const float none = __uint_as_float(0x7FC00000u);       // (a NaN, which does not count)
    float largest = -INFINITY, smallest = INFINITY;
    int n_all = 0;
    each_eight(row, tid, [&](const float *x, int, uint32_t) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool candidate = x[k] >= kLowest;
            const float y = candidate ? x[k] : none;
            n_all += __popcll(__ballot(candidate));
            largest = fmaxf(largest, y);
            smallest = fminf(smallest, y);
        }
    });
    largest = wave_max(largest);
    smallest = -wave_max(-smallest);
    if (lane == 0) { s.largest[wave] = largest; s.smallest[wave] = smallest; s.part_tokens[wave] = n_all; }
    lds_barrier();
    r.top = wave_max(s.largest[lane % kSampleWaves]);
    smallest = -wave_max(-s.smallest[lane % kSampleWaves]);
    r.n_all = wave_sum(lane < kSampleWaves ? s.part_tokens[lane] : 0);
    if (r.n_all == 0) {                        // nothing to draw from
        const int token = first_neg_inf(s, row.logits, row.mask, vocab);
        if (tid == 0) put_draw(b, token, token < 0 ? -(double)INFINITY : 0.0, token < 0 ? 0 : 1, out_tokens, out_logprobs, out_kept);
        return;
    }
    if (r.n_all <= kSampleBlock) {
        each_eight(row, tid, [&](const float *x, int t, uint32_t) {
            uint32_t wanted = 0u;
#pragma unroll
            for (int k = 0; k < 8; ++k) wanted |= (x[k] >= kLowest ? 1u : 0u) << k;
            if (wanted == 0u) return;
            int at = atomicAdd(&s.n_listed, __popc(wanted));
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if ((wanted >> k) & 1u) s.sorted.entry[at++] = (unsigned long long)falling_key(x[k]) << 32 | (uint32_t)(t + k);
        });
        lds_barrier();
        if (r.n_all <= 64) {                   // (by the block: 128 rows of 30 tokens 18.4 us, by one wave 17)
            if (wave == 0) draw_by_wave(lane < r.n_all ? s.sorted.entry[lane] : kNoEntry, r.draw, b, out_tokens, out_logprobs, out_kept, lane);
            return;
        }
        int size = 64;
        while (size < r.n_all) size *= 2;
        draw_sorted<kSampleBlock>(s.sorted, tid < r.n_all ? s.sorted.entry[tid] : kNoEntry, size, r.n_all, r.draw, b, out_tokens, out_logprobs, out_kept, tid);
        return;
    }
    // (2) the bins
    r.infinite = r.top == INFINITY;
    r.binning.set(r.infinite ? 0.0 : (double)r.top, r.infinite ? 0.0 : (double)smallest, r.draw.rate);
    if (r.infinite) {
        int n = 0;
        each_eight(row, tid, [&](const float *x, int, uint32_t) {
#pragma unroll
            for (int k = 0; k < 8; ++k) n += __popcll(__ballot(x[k] == INFINITY));
        });
        if (lane == 0) atomicAdd(&s.weight[0], (unsigned long long)n << kCountShift);
    } else {
        each_eight(row, tid, [&](const float *x, int, uint32_t) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double place = r.binning.place(x[k]);
                if (place < kBinEnd) {
                    const double rounded = place + Binning::kRound;
                    atomicAdd(&s.weight[(uint32_t)__builtin_bit_cast(unsigned long long, rounded)], r.binning.entry(place, rounded));
                }
            }
        });
    }
    lds_barrier();
    constexpr int kPer = kBins / kSampleBlock;
    sum_through<kPer>(s, s.weight, s.tokens, r.infinite ? 1.0 : r.binning.weight(tid * kPer), r.infinite ? 1.0 : r.binning.weight(1), tid);
    // (3) the bins that the places can lie in, by wave 0: lo and hi enclose the weight of what is kept so far
    r.likely = -1;
    if (wave == 0) {
        double lo = s.weight_through(kBins - 1), hi = lo;
        int room = kSampleBlock, n_ranges = 0, likely_from = 0, likely_to = -1;          // likely_from, likely_to: the bins of weights near min_p
        const double unit = r.binning.scale > 0.0 ? 1.0 / r.binning.scale : 0.0;           // of a bin
        auto want = [&](int from, int to) {
            const int n = s.tokens[to] - s.tokens_before(from);
            if (r.infinite || n > room) return;
            room -= n;
            const double m = (double)r.top - 0.5 * (from + to) * unit, h = (0.5 * (to - from) + 0.51) * unit + fabs(m) * 1e-6;
            if (lane == 0) { s.middle[n_ranges] = (float)m; s.half[n_ranges] = (float)h; }
            ++n_ranges;
            for (int i = from + lane; i <= to; i += 64) s.listed[i] = 1;
        };
        if (r.draw.top_k > 0 && r.draw.top_k < min(r.n_all, s.in_bins())) {
            const int bin = s.bin_with(r.draw.top_k, lane);
            if (s.tokens[bin] != r.draw.top_k) want(bin, bin);
            lo = s.weight_before(bin);
            hi = s.weight_through(bin);
        }
        constexpr double kBelow = 1.0 - 1e-9, kAbove = 1.0 + 1e-9;            // beyond what the sums may be off
        if (r.draw.top_p < 1.0) {
            const int from = s.bin_reaching(weight_of_at_least(r.draw.top_p * lo * kBelow), lane), to = s.bin_reaching(weight_of_at_least(r.draw.top_p * hi * kAbove), lane);
            want(from, to);
            lo = fmin(lo, s.weight_before(from));
            hi = fmin(hi, s.weight_through(to));
        }
        if (r.draw.min_p > 0.0 && !r.infinite) {
            const double at = -log(r.draw.min_p) * 1.44269504088896340736 / r.binning.octave;
            if (!(at < kBinEnd - 1.0)) {
                if (s.in_bins() == r.n_all) r.likely = r.n_all;
            } else {
                likely_from = Binning::bin_of(fmax(at - 0.01, 0.0));
                likely_to = Binning::bin_of(fmax(at + 0.01, 0.0));
                want(likely_from, likely_to);
                lo = fmin(lo, s.weight_before(likely_from));
                hi = fmin(hi, s.weight_through(likely_to));
            }
        }
        want(s.bin_reaching(weight_above(r.draw.uniform * lo * kBelow), lane), s.bin_reaching(weight_above(r.draw.uniform * hi * kAbove), lane));
        if (lane == 0) { s.n_ranges = n_ranges; s.likely_from = likely_from; s.likely_to = likely_to; }
    }
    lds_barrier();
    const int n_ranges = __builtin_amdgcn_readfirstlane(s.n_ranges), likely_from = s.likely_from, likely_to = s.likely_to;
    if (n_ranges > 0) {
        float middle[4], half[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            middle[i] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s.middle[i])));
            half[i] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(s.half[i])));
        }
        each_eight<true>(row, tid, [&](const float *x, int t, uint32_t m) {
            bool near[8] = {};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= n_ranges) break;
#pragma unroll
                for (int k = 0; k < 8; ++k) near[k] |= fabsf(x[k] - middle[i]) <= half[i];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (!near[k] || !((m >> k) & 1u)) continue;
                const double place = r.binning.place(x[k]);
                if (place < kBinEnd && s.listed[Binning::bin_of(place)])
                    s.sorted.entry[atomicAdd(&s.n_listed, 1)] = (unsigned long long)falling_key(x[k]) << 32 | (uint32_t)(t + k);
            }
        });
        lds_barrier();
        const int listed = s.n_listed;
        int size = 64;
        while (size < listed) size *= 2;
        const unsigned long long mine = sorted_entry<kSampleBlock>(s.sorted, tid < listed ? s.sorted.entry[tid] : kNoEntry, size, tid);
        auto value_of = [](unsigned long long entry) { return of_falling_key((uint32_t)(entry >> 32)); };
        double upto = 0.0;
        if (wave * 64 < listed) {
            const double w = tid < listed ? draw_weight((double)value_of(mine), (double)r.top, r.draw.rate) : 0.0;
            upto = wave_scan(w);
            if (tid < listed) {
                const int bin = Binning::bin_of(r.binning.place(value_of(mine)));
                if (tid == 0 || Binning::bin_of(r.binning.place(value_of(s.sorted.entry[tid - 1]))) != bin) s.start[bin] = tid;
                if (bin >= likely_from && bin <= likely_to && w >= r.draw.min_p) atomicAdd(&s.likely, 1);
            }
        }
        if (lane == 63) s.sorted.part[wave] = upto;
        lds_barrier();
        const double parts = wave_scan(lane < kSampleWaves ? s.sorted.part[lane] : 0.0);
        if (wave) upto += from_lane(parts, wave - 1);
        s.sorted.upto[tid] = upto;
        lds_barrier();
    }
    // (4) the draw, by wave 0 out of the list
    if (wave == 0) {
        bool known = !(r.draw.min_p > 0.0) || r.likely >= 0;
        if (!known && likely_to >= likely_from) {
            known = true;
            for (int i = likely_from; i <= likely_to; ++i) known &= s.listed[i] != 0;
            if (known) r.likely = s.tokens_before(likely_from) + s.likely;
        }
        bool done = false;
        if (known) {
            const DrawnToken d = draw_from_bins<false>(s, r, row, tid);
            done = d.found && d.by_id;
            if (done && lane == 0) put_draw(b, d.token, d.logprob, d.kept, out_tokens, out_logprobs, out_kept);
        }
        if (lane == 0) {
            s.done = done;
            if (!done) s.row = r;
        }
    }
    lds_barrier();
    if (s.done) return;
    draw_by_block(s, row.logits, row.mask, vocab, b, out_tokens, out_logprobs, out_kept);
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
        hipLaunchKernelGGL(sample_bins_kernel, dim3(batch), dim3(kSampleBlock), 0, stream, static_cast<const uint32_t *>(logits), bitmask, vocab, row_stride,
                           n_words, rows, out_tokens, out_logprobs, out_kept);
    }
    return hipGetLastError();
}

}  // namespace pre3
