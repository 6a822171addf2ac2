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
// Eight numbers of a row to it from element `at` on, as far as it goes.  kWhole: a wave's make whole lines (which may leave the caches at once).
template <class F, bool kWhole>
__device__ __forceinline__ void put_eight(const float x[8], typename F::Stored *row, int at, int n) {
    if (at + 8 <= n) {
        uint16_t *to = reinterpret_cast<uint16_t *>(row + at);
        auto put = [&](uint4 v, int i) {
            if constexpr (kWhole) stream_store(v, to + 8 * i);
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

// out[r][plane][k] = row (row_of ? row_of[r] : r), zeros from k = n on and in the rows from *count (or `rows`) on.
template <class F>
__global__ __launch_bounds__(256) void pack_kernel(const typename F::Stored *in, int64_t in_stride, const int32_t *row_of, const int32_t *count, int rows, int n, char *out, int plane_bytes) {
    const int r = blockIdx.x, group = blockIdx.y * 256 + threadIdx.x;
    if (group * 16 >= plane_bytes) return;
    const bool there = r < (count ? *count : rows);
    float x[8] = {};
    if (there) eight_of<F>(in + (row_of ? row_of[r] : r) * in_stride, group * 8, n, x);
    char *to = out + (int64_t)r * Planes<F>::kCount * plane_bytes + (int64_t)group * 16;
#pragma unroll
    for (int p = 0; p < Planes<F>::kCount; ++p) *reinterpret_cast<uint4 *>(to + (int64_t)p * plane_bytes) = take_plane<F>(x);
}
template <class F>
hipError_t launch_pack(const typename F::Stored *in, int64_t in_stride, const int32_t *row_of, const int32_t *count, int rows, int padded_rows, int n, char *out, int plane_bytes,
                       hipStream_t stream) {
    hipLaunchKernelGGL((pack_kernel<F>), dim3(padded_rows, (plane_bytes / 16 + 255) / 256), dim3(256), 0, stream, in, in_stride, row_of, count, rows, n, out, plane_bytes);
    return hipGetLastError();
}

// out[d][plane][r]: the same transposed, 64 x 64 at a time.  What is not finite becomes 0: the logits that it takes part in have made the slopes
// of their rows NaN already, and the other slopes it is multiplied with are the zeros of tokens that are not allowed.
template <class F>
__global__ __launch_bounds__(256) void pack_transposed_kernel(const typename F::Stored *in, int64_t in_stride, const int32_t *row_of, const int32_t *count, int rows, int n, char *out,
                                                              int plane_bytes) {
    __shared__ __attribute__((aligned(16))) uint16_t tile[64][72];
    const int r0 = blockIdx.x * 64, d0 = blockIdx.y * 64, end = count ? *count : rows;
    float x[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = r0 + h * 32 + threadIdx.x / 8, d = d0 + threadIdx.x % 8 * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[h][i] = 0.0f;
        if (r < end) eight_of<F>(in + (row_of ? row_of[r] : r) * in_stride, d, n, x[h]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(fabsf(x[h][i]) < INFINITY)) x[h][i] = 0.0f;
    }
    for (int p = 0; p < Planes<F>::kCount; ++p) {
        if (p) __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) *reinterpret_cast<uint4 *>(&tile[h * 32 + threadIdx.x / 8][threadIdx.x % 8 * 8]) = take_plane<F>(x[h]);
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int d = h * 32 + threadIdx.x / 8, r = threadIdx.x % 8 * 8;
            if (d0 + d >= n) continue;
            uint32_t v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = tile[r + i][d];
            *reinterpret_cast<uint4 *>(out + ((int64_t)(d0 + d) * Planes<F>::kCount + p) * plane_bytes + (int64_t)(r0 + r) * 2) =
                make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
        }
    }
}
// padded_rows: a multiple of 64, within plane_bytes.
template <class F>
hipError_t launch_pack_transposed(const typename F::Stored *in, int64_t in_stride, const int32_t *row_of, const int32_t *count, int rows, int padded_rows, int n, char *out,
                                  int plane_bytes, hipStream_t stream) {
    hipLaunchKernelGGL((pack_transposed_kernel<F>), dim3((padded_rows + 63) / 64, (n + 63) / 64), dim3(256), 0, stream, in, in_stride, row_of, count, rows, n, out, plane_bytes);
    return hipGetLastError();
}

}  // namespace

}  // namespace pre3
