// gfx950 kernels of a head in 8 bits: the logits of hidden states against weights that are whole numbers of -128 .. 127 with a scale for each
// token.  The hidden states are quantised on the way, a row at a time,
//     s = max |h| / 127,    q_k = h_k * (127 / max |h|)  rounded to the nearest whole number (both steps in 32 bits, halves to even),
//     x_v = (sum of q_k w_vk) s s_v,    -inf where the mask has no bit,
// the sum exact in 32-bit integers, rounded once with its scales and once to the logits' type.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "lanes.hpp"
#include "launch.hpp"
#include "pack.hpp"
#include "product.hpp"
#include "rows.hpp"

namespace pre3 {

namespace {

// A row whose largest number is smaller than this is one of zeros (127 / it would not be a number).
constexpr float kLeastTop = 0x1p-100f;

// A block for every row.  Zeros behind its numbers up to out_bytes.  A row that holds a NaN or an infinity has zeros and a scale of NaN.
template <class F>
__global__ __launch_bounds__(256) void quantise_kernel(const typename F::Stored *in, int64_t in_stride, int rows, int n, int8_t *out, int64_t out_stride, int out_bytes, float *scale) {
    __shared__ float tops[4];
    __shared__ int bads[4];
    const int r = blockIdx.x, tid = threadIdx.x;
    int8_t *to = out + r * out_stride;
    if (r >= rows) {                                                      // (rows that fill a tile)
        for (int at = tid * 8; at < out_bytes; at += 2048) *reinterpret_cast<uint2 *>(to + at) = make_uint2(0, 0);
        return;
    }
    const auto *row = in + r * in_stride;
    constexpr int kHeld = 2;                                              // groups of eight numbers a thread keeps; the others it reads again
    float held[kHeld][8], x[8], top = 0.0f;
    bool bad = false;
    auto see = [&](const float *y) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bad |= !(fabsf(y[e]) < INFINITY);
            top = fmaxf(top, fabsf(y[e]));
        }
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        eight_of<F>(row, min((h * 256 + tid) * 8, (n + 7) / 8 * 8), n, held[h]);
        see(held[h]);
    }
    for (int at = (kHeld * 256 + tid) * 8; at < n; at += 2048) {
        eight_of<F>(row, at, n, x);
        see(x);
    }
    top = wave_max(top);
    bad = __any(bad);
    if (tid % 64 == 0) { tops[tid / 64] = top; bads[tid / 64] = bad; }
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    bad = bads[0] | bads[1] | bads[2] | bads[3];
    const bool none = bad || top < kLeastTop;
    const float factor = none ? 0.0f : 127.0f / top;
    auto put = [&](const float *y, int at) {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int q = none ? 0 : (int)rintf(y[e] * factor);
            w[e / 4] |= (uint32_t)(uint8_t)(int8_t)q << (e % 4 * 8);
        }
        if (at + 8 <= out_bytes) *reinterpret_cast<uint2 *>(to + at) = make_uint2(w[0], w[1]);
        else
            for (int e = 0; at + e < out_bytes; ++e) to[at + e] = (int8_t)(w[e / 4] >> (e % 4 * 8));
    };
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
        const int at = (h * 256 + tid) * 8;
        if (at < out_bytes) put(held[h], at);
    }
    for (int at = (kHeld * 256 + tid) * 8; at < out_bytes; at += 2048) {
        eight_of<F>(row, min(at, (n + 7) / 8 * 8), n, x);
        put(x, at);
    }
    if (tid == 0) scale[r] = bad ? NAN : none ? 0.0f : top / 127.0f;
}

// The tiles of a block.  Those of which no row allows a token have no steps.
template <class Tile>
struct LogitTiles {
    int tiles_m, tiles_n, steps, rows, words;
    const uint32_t *bitmask;
    __device__ bool operator()(int i, TileAt &at) const {
        const int tile = i * gridDim.x + blockIdx.x;
        if (tile >= tiles_m * tiles_n) return false;
        place_of_tile(tile, tiles_m, tiles_n, at.m, at.n);
        at.m0 = at.m * Tile::kM;
        at.n0 = at.n * Tile::kN;
        at.first = 0;
        at.last = steps;
        if (bitmask) {
            constexpr int kWords = Tile::kM / 32;
            bool some = false;                                            // (asked by each wave: the answer is the same in all)
            for (int x = threadIdx.x & 63; x < Tile::kN * kWords; x += 64) {
                const int r = at.n0 + x / kWords, w = at.m0 / 32 + x % kWords;
                if (r < rows && w < words && bitmask[(size_t)r * words + w]) some = true;
                if (__any(some)) break;
            }
            if (!__any(some)) at.last = 0;
        }
        return true;
    }
};

template <class F, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head8_logits_kernel(Operand weight, Operand hidden, int steps, int tiles_m, int tiles_n, const uint32_t *bitmask, int words, int rows,
                                                                      int vocab, const float *row_scale, const float *token_scale, typename F::Stored *out, int64_t out_stride) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    static_assert(Tile::kLaneM == 16, "half a word of the mask");
    Tile tile;
    tile.run(weight, hidden, 1, steps, lds, LogitTiles<Tile>{tiles_m, tiles_n, steps, rows, words, bitmask}, [&](const TileAt &at) {
        const int v = at.m0 + Tile::m_of(0), first = at.n0 + Tile::n_of(0);
        if (v >= vocab) return;
        float by_token[16], by_row[Tile::kNj];
        uint32_t allowed[Tile::kNj];
#pragma unroll
        for (int i = 0; i < 16; ++i) by_token[i] = token_scale[min(v + i, vocab - 1)];
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            const int r = min(first + j, rows - 1);
            by_row[j] = row_scale[r];
            allowed[j] = bitmask ? reinterpret_cast<const uint16_t *>(bitmask + (size_t)r * words)[v >> 4] : 0xFFFFu;
        }
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            if (first + j >= rows) continue;
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = allowed[j] >> i & 1u ? (float)tile.acc[i / 4][j][i % 4] * by_row[j] * by_token[i] : -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; i += 8) put_eight<F, false>(x + i, out + (first + j) * out_stride, v + i, vocab);
        }
    });
}

int tile_rows(int rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }
size_t up(size_t n, size_t to) { return (n + to - 1) / to * to; }

template <class F, class Tile>
hipError_t launch_tile(const Head8Rows &h, const Operand &weight, const Operand &hidden, const float *scale, void *logits, int64_t logits_stride, hipStream_t stream) {
    const int tiles_m = (h.vocab + Tile::kM - 1) / Tile::kM, tiles_n = (h.rows + Tile::kN - 1) / Tile::kN;
    auto *kernel = head8_logits_kernel<F, Tile>;
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), Tile::kLdsBytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(std::min(tiles_m * tiles_n, kUnits * (160 * 1024 / Tile::kLdsBytes))), dim3(Tile::kThreads), Tile::kLdsBytes, stream, weight, hidden, hidden.row_bytes / kStepBytes, tiles_m, tiles_n, h.bitmask,
                       (h.vocab + 31) / 32, h.rows, h.vocab, scale, h.weight_scale, static_cast<typename F::Stored *>(logits), logits_stride);
    return hipGetLastError();
}
template <class F>
hipError_t run(const Head8Rows &h, void *logits, int64_t logits_stride, void *workspace, hipStream_t stream) {
    const int n_tile = tile_rows(h.rows), padded = (int)up(h.rows, n_tile), bytes = (int)up(h.dim, kStepBytes);
    auto *q = static_cast<int8_t *>(workspace);
    auto *scale = reinterpret_cast<float *>(q + (size_t)padded * bytes);
    hipLaunchKernelGGL((quantise_kernel<F>), dim3(padded), dim3(256), 0, stream, static_cast<const typename F::Stored *>(h.hidden), h.hidden_stride, h.rows, h.dim, q, (int64_t)bytes, bytes,
                       scale);
    const Operand hidden{reinterpret_cast<const char *>(q), bytes, padded, bytes, 0},
        weight{reinterpret_cast<const char *>(h.weight), h.weight_stride, h.vocab, (int)up(h.dim, 16), 0};
    switch (n_tile) {
        case 32: return launch_tile<F, ProductTile<ProductI8, 128, 32, 2, 1, 4>>(h, weight, hidden, scale, logits, logits_stride, stream);
        case 64: return launch_tile<F, ProductTile<ProductI8, 256, 64, 4, 1, 3>>(h, weight, hidden, scale, logits, logits_stride, stream);
        case 128: return launch_tile<F, ProductTile<ProductI8, 256, 128, 4, 2, 3>>(h, weight, hidden, scale, logits, logits_stride, stream);
        default: return launch_tile<F, ProductTile<ProductI8, 256, 256, 4, 2, 2>>(h, weight, hidden, scale, logits, logits_stride, stream);
    }
}

}  // namespace

size_t head8_workspace_bytes(int rows, int dim) {
    const size_t padded = up(rows, tile_rows(rows));
    return padded * up(dim, kStepBytes) + padded * 4;
}
hipError_t launch_head8(const Head8Rows &h, void *logits, int64_t logits_stride, void *workspace, hipStream_t stream) {
    switch (h.type) {
        case kLogitBf16: return run<LogitsBf16>(h, logits, logits_stride, workspace, stream);
        case kLogitF16: return run<LogitsF16>(h, logits, logits_stride, workspace, stream);
        default: return run<LogitsF32>(h, logits, logits_stride, workspace, stream);
    }
}

hipError_t launch_quantise(const void *in, LogitType type, int64_t in_stride, int rows, int dim, int8_t *out, int64_t out_stride, float *scale, hipStream_t stream) {
    auto go = [&](auto type_of) {
        typedef decltype(type_of) F;
        hipLaunchKernelGGL((quantise_kernel<F>), dim3(rows), dim3(256), 0, stream, static_cast<const typename F::Stored *>(in), in_stride, rows, dim, out, out_stride, (int)up(dim, 16), scale);
        return hipGetLastError();
    };
    return type == kLogitBf16 ? go(LogitsBf16()) : type == kLogitF16 ? go(LogitsF16()) : go(LogitsF32());
}

}  // namespace pre3
