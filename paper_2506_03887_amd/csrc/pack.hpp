// Operands of a product out of matrices as callers have them: rows of any stride, alignment and length, of one of three types, become rows of
// 16-bit numbers at 16-byte boundaries, zeros behind them; 32-bit numbers become three planes of bf16 numbers side by side, whose sum they are.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rows.hpp"

namespace pre3 {

namespace {

// What a number's planes are made of, plane by plane.
template <class F>
struct Planes {
    static constexpr int kCount = 1;
    typedef F Part;
};
template <>
struct Planes<LogitsF32> {
    static constexpr int kCount = 3;
    typedef LogitsBf16 Part;
};

// Eight numbers of a row from element `at` on, zeros beyond `n`.
template <class F>
__device__ __forceinline__ void eight_of(const typename F::Stored *row, int at, int n, float x[8]) {
    if (at + 8 <= n) {
        const Eight<F> e = load_eight<F, false>(row, at / 8);
        if constexpr (sizeof(typename F::Stored) == 2) {
            const uint32_t w[4] = {e.v[0].x, e.v[0].y, e.v[0].z, e.v[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = F::value(w[i] & 0xFFFFu);
                x[2 * i + 1] = F::value(w[i] >> 16);
            }
        } else {
            const uint32_t w[8] = {e.v[0].x, e.v[0].y, e.v[0].z, e.v[0].w, e.v[1].x, e.v[1].y, e.v[1].z, e.v[1].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = F::value(w[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = at + i < n ? F::value(row[at + i]) : 0.0f;
    }
}
// And back, as they lie in memory.
template <class F>
__device__ __forceinline__ Eight<F> eight_from(const float x[8]) {
    Eight<F> e;
    if constexpr (sizeof(typename F::Stored) == 2) e.v[0] = make_uint4(F::pair(x[0], x[1]), F::pair(x[2], x[3]), F::pair(x[4], x[5]), F::pair(x[6], x[7]));
    else {
        e.v[0] = make_uint4(F::pattern(x[0]), F::pattern(x[1]), F::pattern(x[2]), F::pattern(x[3]));
        e.v[1] = make_uint4(F::pattern(x[4]), F::pattern(x[5]), F::pattern(x[6]), F::pattern(x[7]));
    }
    return e;
}
// Eight numbers of a row to it from element `at` on, as far as it goes.  kWhole: eight 16-bit numbers of each lane of a wave make whole lines (which may
// leave the caches at once; parts of lines have to meet there first, 256 x 256 f16 results of rows of 1,001 276 and 121 us).
template <class F, bool kWhole>
__device__ __forceinline__ void put_eight(const float x[8], typename F::Stored *row, int at, int n) {
    if (at + 8 <= n) {
        uint16_t *to = reinterpret_cast<uint16_t *>(row + at);
        auto put = [&](uint4 v, int i) {
            if constexpr (kWhole && sizeof(typename F::Stored) == 2) stream_store(v, to + 8 * i);
            else *reinterpret_cast<UnalignedUint4 *>(to + 8 * i) = UnalignedUint4{v.x, v.y, v.z, v.w};
        };
        if constexpr (sizeof(typename F::Stored) == 2) {
            put(make_uint4(F::pair(x[0], x[1]), F::pair(x[2], x[3]), F::pair(x[4], x[5]), F::pair(x[6], x[7])), 0);
        } else {
            put(make_uint4(F::pattern(x[0]), F::pattern(x[1]), F::pattern(x[2]), F::pattern(x[3])), 0);
            put(make_uint4(F::pattern(x[4]), F::pattern(x[5]), F::pattern(x[6]), F::pattern(x[7])), 1);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e < n) row[at + e] = (typename F::Stored)F::pattern(x[e]);
    }
}
// Their parts in one plane; x becomes what is left.
template <class F>
__device__ __forceinline__ uint4 take_plane(float x[8]) {
    typedef typename Planes<F>::Part P;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = P::pair(x[2 * i], x[2 * i + 1]);
        if constexpr (Planes<F>::kCount > 1) {
            x[2 * i] -= P::value(w[i] & 0xFFFFu);
            x[2 * i + 1] -= P::value(w[i] >> 16);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Rows to be packed: those of a matrix [rows][n] or, with row_of, *count of them by their numbers.
struct Pack {
    const void *in;
    int64_t stride;
    const int32_t *row_of, *count;             // null: all rows, in order
    int rows, n;
    int padded;                                // rows that are written, zeros behind the last one
    char *out;                                 // [row][plane][n, zeros to the plane's end], null: not wanted
    int plane_bytes;                           // a multiple of 16
};
__host__ __device__ inline int pack_blocks(const Pack &p) { return p.out ? (int)(((int64_t)p.padded * (p.plane_bytes / 16) + 255) / 256) : 0; }

// Eight numbers a thread, of one of two matrices.
template <class F>
__global__ __launch_bounds__(256) void pack_kernel(Pack one, Pack two) {
    constexpr int kPlanes = Planes<F>::kCount;
    const int first = pack_blocks(one);
    const Pack &p = (int)blockIdx.x < first ? one : two;
    const int64_t at = (int64_t)((int)blockIdx.x < first ? blockIdx.x : blockIdx.x - first) * 256 + threadIdx.x;
    const int groups = p.plane_bytes / 16, r = (int)(at / groups), group = (int)(at % groups);
    if (r >= p.padded) return;
    float x[8] = {};
    if (r < (p.count ? *p.count : p.rows)) eight_of<F>(static_cast<const typename F::Stored *>(p.in) + (p.row_of ? p.row_of[r] : r) * p.stride, group * 8, p.n, x);
    char *to = p.out + (int64_t)r * kPlanes * p.plane_bytes + (int64_t)group * 16;
#pragma unroll
    for (int plane = 0; plane < kPlanes; ++plane) *reinterpret_cast<uint4 *>(to + (int64_t)plane * p.plane_bytes) = take_plane<F>(x);
}
template <class F>
hipError_t launch_pack(const Pack &one, const Pack &two, hipStream_t stream) {
    const int blocks = pack_blocks(one) + pack_blocks(two);
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL((pack_kernel<F>), dim3(blocks), dim3(256), 0, stream, one, two);
    return hipGetLastError();
}

}  // namespace

}  // namespace pre3
