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
    int padded;                                // rows that are written (transposed: numbers of a row), a multiple of 64: zeros behind the last one
    char *rows_out, *transposed;               // [row][plane][n, zeros to a multiple of 64] and [n][plane][row], null: not wanted
    int rows_plane, transposed_plane;          // bytes
};
constexpr int kPackSide = 64;
__host__ __device__ inline int pack_tiles(const Pack &p) { return p.rows_out || p.transposed ? p.padded / kPackSide * ((p.n + kPackSide - 1) / kPackSide) : 0; }

// 64 x 64 numbers of one of two matrices.  In what is transposed, a number that is not finite becomes 0: the logits that it takes part in have made the
// slopes of their rows NaN already, and the other slopes it is multiplied with are the zeros of tokens that are not allowed.
// (4,096 x 1,001 f16 of 100,003 rows, both ways: 600 MB at 4.9 TB/s)
template <class F>
__global__ __launch_bounds__(256) void pack_kernel(Pack one, Pack two) {
    __shared__ __attribute__((aligned(16))) uint16_t tile[kPackSide][72];
    constexpr int kPlanes = Planes<F>::kCount;
    const int first = pack_tiles(one), block = blockIdx.x;
    const Pack &p = block < first ? one : two;
    const int at = block < first ? block : block - first, tiles_n = (p.n + kPackSide - 1) / kPackSide, r0 = at / tiles_n * kPackSide, d0 = at % tiles_n * kPackSide;
    const int end = p.count ? *p.count : p.rows, column = threadIdx.x % 8 * 8;
    float x[2][8];
    uint32_t bad[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = r0 + h * 32 + threadIdx.x / 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[h][i] = 0.0f;
        if (r < end) eight_of<F>(static_cast<const typename F::Stored *>(p.in) + (p.row_of ? p.row_of[r] : r) * p.stride, d0 + column, p.n, x[h]);
        bad[h] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(fabsf(x[h][i]) < INFINITY)) bad[h] |= 1u << i;
    }
    for (int plane = 0; plane < kPlanes; ++plane) {
        if (plane && p.transposed) __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = h * 32 + threadIdx.x / 8;
            uint4 w = take_plane<F>(x[h]);
            if (p.rows_out) *reinterpret_cast<uint4 *>(p.rows_out + ((int64_t)(r0 + r) * kPlanes + plane) * p.rows_plane + (d0 + column) * 2) = w;
            if (!p.transposed) continue;
            if (bad[h]) {
                uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (bad[h] >> i & 1u) v[i / 2] &= i % 2 ? 0xFFFFu : 0xFFFF0000u;
                w = make_uint4(v[0], v[1], v[2], v[3]);
            }
            *reinterpret_cast<uint4 *>(&tile[r][column]) = w;
        }
        if (!p.transposed) continue;
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int d = h * 32 + threadIdx.x / 8, r = threadIdx.x % 8 * 8;
            if (d0 + d >= p.n) continue;
            uint32_t v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = tile[r + i][d];
            *reinterpret_cast<uint4 *>(p.transposed + ((int64_t)(d0 + d) * kPlanes + plane) * p.transposed_plane + (int64_t)(r0 + r) * 2) =
                make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
        }
    }
}
template <class F>
hipError_t launch_pack(const Pack &one, const Pack &two, hipStream_t stream) {
    const int blocks = pack_tiles(one) + pack_tiles(two);
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL((pack_kernel<F>), dim3(blocks), dim3(256), 0, stream, one, two);
    return hipGetLastError();
}

}  // namespace

}  // namespace pre3
