// A row of logits of one of three types behind its mask, and a pass over it.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "argmax.hpp"
#include "stream_access.hpp"

namespace pre3 {

namespace {

// Logits of one type: a number from its pattern, and patterns from numbers, rounded to the nearest.
struct LogitsBf16 {
    typedef uint16_t Stored;
    __device__ static float value(uint32_t h) { return __uint_as_float(h << 16); }
    __device__ static uint32_t pattern(float x) {
        const __bf16 y = (__bf16)x;
        return __builtin_bit_cast(uint16_t, y);
    }
    __device__ static uint32_t pair(float lo, float hi) {
        typedef __bf16 Two __attribute__((ext_vector_type(2)));
        typedef float Floats __attribute__((ext_vector_type(2)));
        const Floats x = {lo, hi};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, Two));
    }
    static constexpr uint32_t kNegInf = 0xFF80u;
};
struct LogitsF16 {
    typedef uint16_t Stored;
    __device__ static float value(uint32_t h) { return (float)__builtin_bit_cast(_Float16, (uint16_t)h); }
    __device__ static uint32_t pattern(float x) {
        const _Float16 y = (_Float16)x;
        return __builtin_bit_cast(uint16_t, y);
    }
    __device__ static uint32_t pair(float lo, float hi) { return pattern(lo) | pattern(hi) << 16; }
    static constexpr uint32_t kNegInf = 0xFC00u;
};
struct LogitsF32 {
    typedef uint32_t Stored;
    __device__ static float value(uint32_t h) { return __uint_as_float(h); }
    __device__ static uint32_t pattern(float x) { return __float_as_uint(x); }
    static constexpr uint32_t kNegInf = 0xFF800000u;
};

// Eight neighbouring logits as they are stored.
template <class F>
struct Eight { uint4 v[sizeof(typename F::Stored) / 2]; };
typedef NativeUint4 __attribute__((aligned(2))) UnalignedUint4;
// kLast: the row is not read again (the line may leave the caches first).
template <class F, bool kLast>
__device__ __forceinline__ Eight<F> load_eight(const typename F::Stored *row, int g) {
    Eight<F> e;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(e) / 16); ++i) {
        const char *at = reinterpret_cast<const char *>(row) + ((size_t)(uint32_t)g * sizeof(e) + i * 16);
        if (kLast) e.v[i] = stream_load(reinterpret_cast<const uint16_t *>(at));
        else {
            const UnalignedUint4 x = *reinterpret_cast<const UnalignedUint4 *>(at);
            e.v[i] = make_uint4(x.x, x.y, x.z, x.w);
        }
    }
    return e;
}
// Their values; -inf where the mask byte has no bit.
template <class F>
__device__ __forceinline__ void values_of(const Eight<F> &e, uint32_t allowed, const uint2 *table, float x[8]) {
    if constexpr (sizeof(typename F::Stored) == 2) {
        const uint4 allow = expand_mask_byte(table, allowed);
        constexpr uint32_t kNone = F::kNegInf | F::kNegInf << 16;
        const uint32_t w[4] = {e.v[0].x, e.v[0].y, e.v[0].z, e.v[0].w}, a[4] = {allow.x, allow.y, allow.z, allow.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t y = (w[i] & a[i]) | (kNone & ~a[i]);
            x[2 * i] = F::value(y & 0xFFFFu);
            x[2 * i + 1] = F::value(y >> 16);
        }
    } else {
        const uint32_t w[8] = {e.v[0].x, e.v[0].y, e.v[0].z, e.v[0].w, e.v[1].x, e.v[1].y, e.v[1].z, e.v[1].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (allowed >> i) & 1u ? F::value(w[i]) : -INFINITY;
    }
}
// What a row's kernels get.
template <class F>
struct Row {
    const typename F::Stored *logits;
    const uint32_t *mask;                      // null: every token is allowed
    int vocab;
    __device__ bool allows(int t) const { return !mask || ((mask[t >> 5] >> (t & 31)) & 1u); }
    __device__ float value(int t) const { return F::value(logits[t]); }
};

// Groups of eight in a thread's hands at a time, and as many on their way.  (Four of 16 bits took the registers that the list needs:
// the forward pass on 2,048 x 32,000 37 us, 28 with two; loss and gradient of 4,096 x 128,256 456 and 429.)
constexpr int kUnroll = 2;

// One pass over the groups `from` .. `to` of a row, kUnroll of them at a time and a thread, the next ones on their way while fn(group,
// its logits, its mask byte) sees the present ones.  Groups of which nothing is allowed are not fetched (their lanes ask for the first one).
// go(): called with the first ones on their way; false ends the pass.
template <int kBlock, class F, bool kLast, class Go, class Fn>
__device__ __forceinline__ void each_group(const Row<F> &row, int from, int to, int tid, Go go, Fn fn) {
    constexpr int kU = kUnroll;
    const uint8_t *mask = reinterpret_cast<const uint8_t *>(row.mask);
    Eight<F> now[kU], next[kU];
    uint32_t m_now[kU], m_next[kU], m_after[kU];
    auto load_mask = [&](int g0, uint32_t *m) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int g = g0 + u * kBlock;
            m[u] = mask ? mask[min(g, to - 1)] : 0xFFu;
            if (g >= to) m[u] = 0u;
        }
    };
    auto load = [&](int g0, const uint32_t *m, Eight<F> *e) {
#pragma unroll
        for (int u = 0; u < kU; ++u) e[u] = load_eight<F, kLast>(row.logits, m[u] ? g0 + u * kBlock : from);
    };
    if (from >= to) { go(); return; }
    int g = from + tid;
    load_mask(g, m_now);
    load_mask(g + kU * kBlock, m_next);
    load(g, m_now, now);
    if (!go()) return;
    for (int g0 = from; g0 < to; g0 += kU * kBlock, g += kU * kBlock) {
        load_mask(g + 2 * kU * kBlock, m_after);
        load(g + kU * kBlock, m_next, next);
        fn(g, now, m_now);
#pragma unroll
        for (int u = 0; u < kU; ++u) { now[u] = next[u]; m_now[u] = m_next[u]; m_next[u] = m_after[u]; }
    }
}

}  // namespace

}  // namespace pre3
