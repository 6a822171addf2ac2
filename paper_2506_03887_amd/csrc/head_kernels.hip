// gfx950 kernels of a head's cross entropy: the loss of one target token a row in the logits  x = hidden weight^T  behind the token mask, and
// its gradients.  With p = softmax(x) over a row's allowed tokens, t its target and g the gradient of what is minimised with respect to
// its loss,
//     loss = log(sum of exp x) - x_t,      s_v = g (p_v - [v = t]),      d hidden = s weight,      d weight = s^T hidden.
// A row without a target, or whose target the mask leaves out, has no loss and no gradient: such rows are not computed at all, the others
// lie side by side in what the products read.
//
// The logits are never kept.  The forward pass leaves of a tile of logits its rows' maxima and sums of exponentials.  The backward pass makes
// the logits of a piece of the vocabulary again, writes their slopes s in the operands' type, along the vocabulary and along the rows, and
// multiplies them into both gradients: four products of 2 rows x vocabulary x dim operations each, where keeping the logits would take
// three and 2 to 4 bytes for every logit.
//
// Slopes are rounded to the operands' type: bf16 to 2^-8 of themselves at most, as the gradients they make are rounded after that; f16, whose range would
// lose the small ones, after a common power of two that brings the largest weight of a row to 2^14.  Sums are held in 32 bits.  32-bit operands and
// slopes are the sums of three bf16 numbers, of 8 bits each, and a product of two is the six products of parts that reach its 24
// bits (2 x 6 operations instead of 2, at 16 times the rate of 32-bit matrix instructions).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "launch.hpp"
#include "lanes.hpp"
#include "pack.hpp"
#include "product.hpp"
#include "rows.hpp"

namespace pre3 {

namespace {

constexpr float kLog2E = 1.44269504088896340736f;

// What the rows' kernel finds out for all others: the rows that have a target ("taught"), side by side.
struct Taught {
    int32_t *count;                // [1]
    float *scale;                  // [2]: of the slopes, and its inverse
    int32_t *place;                // [rows]: where a row lies among them, -1: not taught
    int32_t *row;                  // [rows]: and back
    int32_t *target;               // [rows], by place
    float *weight;                 // [rows], by place
};

__device__ __forceinline__ int64_t id_at(const void *ids, int bytes, int i) {
    return bytes == 8 ? static_cast<const int64_t *>(ids)[i] : static_cast<const int32_t *>(ids)[i];
}

// One block: which rows are taught.  With row_weight also the power of two for f16 slopes.
constexpr int kRowsThreads = 1024;
__global__ __launch_bounds__(kRowsThreads) void head_rows_kernel(const void *targets, int target_bytes, const uint32_t *bitmask, int rows, int vocab, Taught taught,
                                                                 bool weighted, const float *row_weight, int64_t weight_stride, bool scaled) {
    __shared__ int sums[kRowsThreads / 64];
    __shared__ float most[kRowsThreads / 64];
    constexpr int kEach = 4;                                              // rows of a thread, side by side
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, words = (vocab + 31) / 32;
    int before = 0;
    float top = 0.0f;
    for (int r0 = 0; r0 < rows; r0 += kRowsThreads * kEach) {
        const int first = r0 + tid * kEach;
        int target[kEach], mine = 0;
        float g[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int r = first + i;
            const int64_t t = r < rows ? id_at(targets, target_bytes, r) : -1;
            target[i] = t >= 0 && t < vocab ? (int)t : -1;
            g[i] = weighted && row_weight && r < rows ? row_weight[(int64_t)r * weight_stride] : 1.0f;
        }
        if (bitmask) {
            uint32_t word[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) word[i] = target[i] >= 0 ? bitmask[(size_t)(first + i) * words + (target[i] >> 5)] : 0u;
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (!(word[i] >> (target[i] & 31) & 1u)) target[i] = -1;
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) mine += target[i] >= 0;
        const int upto = (int)wave_scan((uint32_t)mine);
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        int at = before + upto - mine;
        for (int w = 0; w < kRowsThreads / 64; ++w) {
            if (w < wave) at += sums[w];
            before += sums[w];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (first + i < rows) taught.place[first + i] = target[i] >= 0 ? at : -1;
            if (target[i] < 0) continue;
            taught.row[at] = first + i;
            taught.target[at] = target[i];
            if (weighted) {
                taught.weight[at] = g[i];
                if (fabsf(g[i]) < INFINITY) top = fmaxf(top, fabsf(g[i]));
            }
            ++at;
        }
    }
    if (tid == 0) *taught.count = before;
    if (!weighted) return;
    top = wave_max(top);
    if (lane == 0) most[wave] = top;
    __syncthreads();
    if (tid != 0) return;
    for (int w = 1; w < kRowsThreads / 64; ++w) top = fmaxf(top, most[w]);
    // 2^14 / 2^(exponent of the largest weight): slopes of up to 2^15 in f16, normal numbers down to 2^-28 of the largest
    int e = scaled && top > 0.0f ? 14 - ilogbf(top) : 0;
    e = min(max(e, -100), 100);
    taught.scale[0] = ldexpf(1.0f, e);
    taught.scale[1] = ldexpf(1.0f, -e);
}

// What a tile's kernels know of the tokens' side.
struct HeadMask {
    const uint32_t *bitmask;       // null: every token is allowed
    int vocab, words;
};
// A lane's share of a tile: 16 tokens of each of its rows.
constexpr int kLaneTokens = 16;
// Which of the 16 from `v` on (a multiple of 16) are allowed in a row.
__device__ __forceinline__ uint32_t allowed_bits(const HeadMask &mask, int row, int v) {
    const int left = mask.vocab - v;
    if (left <= 0) return 0u;
    const uint32_t there = left >= kLaneTokens ? 0xFFFFu : (1u << left) - 1u;
    return mask.bitmask ? there & reinterpret_cast<const uint16_t *>(mask.bitmask + (size_t)row * mask.words)[v >> 4] : there;
}
// The tiles of a block over the taught rows, and of a piece's tokens.  kToStep: rows behind the last one as well, to the end of its step along the rows;
// tiles of nothing else have no steps.
constexpr int kStepRows = kStepBytes / 2;
template <class Tile, bool kToStep>
struct RowTiles {
    int rows, tiles_m, tiles_n, steps;
    __device__ RowTiles(int tiles_m_, int rows_, int steps_)
        : rows(rows_), tiles_m(tiles_m_), tiles_n(((kToStep ? (rows + kStepRows - 1) / kStepRows * kStepRows : rows) + Tile::kN - 1) / Tile::kN), steps(steps_) {}
    __device__ bool operator()(int i, TileAt &at) const {
        const int tile = i * gridDim.x + blockIdx.x;
        if (tile >= tiles_m * tiles_n) return false;
        place_of_tile(tile, tiles_m, tiles_n, at.m, at.n);
        at.m0 = at.m * Tile::kM;
        at.n0 = at.n * Tile::kN;
        at.first = 0;
        at.last = at.n0 < rows ? steps : 0;
        return true;
    }
};

// Tokens of a wave's share of a tile.
constexpr int kPartTokens = 64;

// Maximum, and sum of the exponentials over it, of every taught row over a wave's share of a tile's tokens; a target's logit.
template <class T, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head_stats_kernel(Operand weight, Operand hidden, int pairs, int steps, int v0, int tiles_m, HeadMask mask, const int32_t *count,
                                                                    const int32_t *row_of, const int32_t *target_of, float2 *parts, int parts_stride, float *target_logit) {
    static_assert(Tile::kLaneM == kLaneTokens && Tile::kM / Tile::kWavesM == kPartTokens, "a lane's tokens");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int rows = *count;
    Tile tile;
    tile.run(weight, hidden, pairs, lds, RowTiles<Tile, false>(tiles_m, rows, steps), [&](const TileAt &at) {
        const int v = v0 + at.m0 + Tile::m_of(), first = at.n0 + Tile::n_of();
        float2 *out = parts + (size_t)((v0 + at.m0) / kPartTokens + Tile::wave() / Tile::kWavesN) * parts_stride;
        uint32_t allowed[Tile::kNj];
        int target[Tile::kNj];
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            const int n = min(first + j, rows - 1);
            target[j] = target_of[n] - v;                                 // within the share: whose logit is wanted
            allowed[j] = allowed_bits(mask, row_of[n], v);
        }
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            const bool there = first + j < rows;
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < Tile::kMi; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (target[j] == i * 4 + e && there) target_logit[first + j] = tile.acc[i][j][e];
                    if (!(allowed[j] >> (i * 4 + e) & 1u)) tile.acc[i][j][e] = -INFINITY;
                    top = fmaxf(top, tile.acc[i][j][e]);
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < Tile::kMi; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((tile.acc[i][j][e] - base) * kLog2E);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (Tile::lane() < 16 && there) out[first + j] = make_float2(top, sum);
        }
    });
}

// A row's parts joined, kRows rows to a block, in one pass: the sums, over the largest maximum so far, in 64 bits.
struct Joined { float top; double sum; };
__device__ __forceinline__ Joined join(Joined a, float top, double sum) {
    const float most = fmaxf(a.top, top);
    if (most == -INFINITY) return {most, a.sum + sum};                    // (nothing yet, or a NaN)
    return {most, a.sum * __builtin_amdgcn_exp2f((a.top - most) * kLog2E) + sum * __builtin_amdgcn_exp2f((top - most) * kLog2E)};
}
template <int kRows>
__global__ __launch_bounds__(1024) void head_join_kernel(const int32_t *place, int rows, const float2 *parts, int parts_stride, int n_parts, const float *target_logit, float *loss,
                                                         float2 *stats) {
    constexpr int kOver = 1024 / kRows;                                   // threads of a row
    __shared__ Joined joined[kOver][kRows];
    const int i = threadIdx.x % kRows, part = threadIdx.x / kRows, r = blockIdx.x * kRows + i;
    const int at = r < rows ? place[r] : -1;
    Joined all = {-INFINITY, 0.0};
    if (at >= 0)
        for (int p = part; p < n_parts; p += kOver) {
            const float2 x = parts[(size_t)p * parts_stride + at];
            all = join(all, x.x, x.y);
        }
    joined[part][i] = all;
    for (int half = kOver / 2; half > 0; half /= 2) {
        __syncthreads();
        if (part < half) joined[part][i] = join(joined[part][i], joined[part + half][i].top, joined[part + half][i].sum);
    }
    if (part || r >= rows) return;
    all = joined[0][i];
    if (loss) loss[r] = at < 0 ? 0.0f : (float)(log(all.sum) + ((double)all.top - (double)target_logit[at]));
    if (stats) stats[r] = at < 0 ? make_float2(0.0f, 1.0f) : make_float2(all.top, (float)all.sum);
}

// Numbers of 16 bits side by side, in pieces of at most 16 bytes.
template <class F, int kCount>
__device__ __forceinline__ void put_16_bit(const float *x, char *to) {
    uint32_t w[kCount / 2];
#pragma unroll
    for (int i = 0; i < kCount / 2; ++i) w[i] = F::pair(x[2 * i], x[2 * i + 1]);
    if constexpr (kCount == 2) *reinterpret_cast<uint32_t *>(to) = w[0];
    else if constexpr (kCount == 4) *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
    else
#pragma unroll
        for (int i = 0; i < kCount / 8; ++i) *reinterpret_cast<uint4 *>(to + 16 * i) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}

// The slopes of a piece of the vocabulary, as numbers of 16 bits in one to three planes: [row][plane][token] and [token][plane][row], zeros from the last
// taught row to the end of its step.
struct Slopes {
    char *by_row, *by_token;       // null: not wanted
    int64_t row_stride, token_stride;
    int row_plane, token_plane;
};
template <class T, class F, class Tile, int kPlanes>
__global__ __launch_bounds__(Tile::kThreads) void head_slopes_kernel(Operand weight, Operand hidden, int pairs, int steps, int v0, int tiles_m, HeadMask mask, Taught taught,
                                                                     const float2 *stats, Slopes out) {
    static_assert(Tile::kLaneM == kLaneTokens && Tile::kM / Tile::kWavesM == kPartTokens, "a lane's tokens");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int rows = *taught.count;
    const float scale = taught.scale[0];
    Tile tile;
    tile.run(weight, hidden, pairs, lds, RowTiles<Tile, true>(tiles_m, rows, steps), [&](const TileAt &at) {
        const int m = at.m0 + Tile::m_of(), v = v0 + m, first = at.n0 + Tile::n_of();
        uint32_t allowed[Tile::kNj];
        int target[Tile::kNj];
        float g[Tile::kNj], share[Tile::kNj], top[Tile::kNj];
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            const int n = min(first + j, rows - 1), row = taught.row[n];
            const float2 sum = stats[row];
            target[j] = taught.target[n] - v;
            allowed[j] = first + j < rows ? allowed_bits(mask, row, v) : 0u;
            g[j] = taught.weight[n] * scale;
            top[j] = sum.x;
            share[j] = 1.0f / sum.y;
        }
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j)
#pragma unroll
            for (int i = 0; i < Tile::kMi; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float p = __builtin_amdgcn_exp2f((tile.acc[i][j][e] - top[j]) * kLog2E) * share[j];
                    if (target[j] == i * 4 + e) p -= 1.0f;
                    tile.acc[i][j][e] = allowed[j] >> (i * 4 + e) & 1u ? p * g[j] : 0.0f;
                }
#pragma unroll
        for (int plane = 0; plane < kPlanes; ++plane) {
            if (out.by_row)
#pragma unroll
                for (int j = 0; j < Tile::kNj; ++j) {
                    float x[kLaneTokens];
#pragma unroll
                    for (int i = 0; i < kLaneTokens; ++i) x[i] = tile.acc[i / 4][j][i % 4];
                    put_16_bit<F, kLaneTokens>(x, out.by_row + (first + j) * out.row_stride + (int64_t)plane * out.row_plane + m * 2);
                }
            if (out.by_token)
#pragma unroll
                for (int i = 0; i < kLaneTokens; ++i) {
                    float x[Tile::kNj];
#pragma unroll
                    for (int j = 0; j < Tile::kNj; ++j) x[j] = tile.acc[i / 4][j][i % 4];
                    put_16_bit<F, Tile::kNj>(x, out.by_token + (m + i) * out.token_stride + (int64_t)plane * out.token_plane + first * 2);
                }
            if (plane + 1 < kPlanes)                                      // what is left for the next plane
#pragma unroll
                for (int j = 0; j < Tile::kNj; ++j)
#pragma unroll
                    for (int i = 0; i < Tile::kMi; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) tile.acc[i][j][e] -= F::value(F::pattern(tile.acc[i][j][e]));
        }
    });
}

// d hidden of the taught rows, over a piece of the vocabulary: sums[split][row][dim], of which each split takes its share of the piece's steps.
template <class T, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head_hidden_grad_kernel(Operand weight_t, Operand slopes, int pairs, int steps, int splits, int tiles_m, const int32_t *count, float *sums,
                                                                          int sums_stride, int sums_rows, bool first) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    static_assert(Tile::kLaneM == kLaneTokens, "a lane's numbers");
    const int tiles_n = (*count + Tile::kN - 1) / Tile::kN;
    auto tiles = [&](int i, TileAt &at) {
        const int t = i * gridDim.x + blockIdx.x;
        if (t >= tiles_m * splits * tiles_n) return false;
        place_of_tile(t, tiles_m * splits, tiles_n, at.m, at.n);
        const int split = at.m / tiles_m;
        at.m0 = (at.m - split * tiles_m) * Tile::kM;
        at.n0 = at.n * Tile::kN;
        constexpr int kEach = kStepBytes / Tile::kStep;                   // (whole steps of the longest kind)
        at.first = steps * split / splits * kEach;
        at.last = steps * (split + 1) / splits * kEach;
        return true;
    };
    Tile tile;
    tile.run(weight_t, slopes, pairs, lds, tiles, [&](const TileAt &at) {
        const int d = at.m0 + Tile::m_of();
        float *out = sums + ((size_t)(at.m / tiles_m) * sums_rows + at.n0 + Tile::n_of()) * sums_stride + d;
        if (d >= sums_stride) return;                                     // (a multiple of 16)
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            Float4 *to = reinterpret_cast<Float4 *>(out + (size_t)j * sums_stride);
            Float4 sum[Tile::kMi];
#pragma unroll
            for (int i = 0; i < Tile::kMi; ++i) sum[i] = first ? Float4{0, 0, 0, 0} : to[i];
#pragma unroll
            for (int i = 0; i < Tile::kMi; ++i) to[i] = sum[i] + tile.acc[i][j];
        }
    });
}
// Every row of d hidden from the splits' sums, rounded once; zeros for rows that are not taught.
template <class F>
__global__ __launch_bounds__(256) void head_hidden_join_kernel(const int32_t *place, const float *scale, const float *sums, int splits, int sums_stride, int sums_rows, int dim,
                                                               typename F::Stored *out, int64_t out_stride) {
    const int r = blockIdx.x, at = place[r];
    const float back = scale[1];
    for (int d = blockIdx.y * 1024 + threadIdx.x * 4, end = min(dim, (int)(blockIdx.y + 1) * 1024); d < end; d += 1024) {
        Float4 x = {0, 0, 0, 0};
        if (at >= 0) {
            for (int s = 0; s < splits; ++s) x += *reinterpret_cast<const Float4 *>(sums + ((size_t)s * sums_rows + at) * sums_stride + d);
            x *= back;
        }
        for (int e = 0; e < 4 && d + e < dim; ++e) out[r * out_stride + d + e] = (typename F::Stored)F::pattern(x[e]);
    }
}

// d weight of a piece of the vocabulary, whole: out[token][dim].
template <class T, class F, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head_weight_grad_kernel(Operand hidden_t, Operand slopes, int pairs, int tiles_m, int tiles_n, const int32_t *count, const float *scale,
                                                                          int dim, int tokens, typename F::Stored *out, int64_t out_stride) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int steps = (*count + kStepRows - 1) / kStepRows * (kStepBytes / Tile::kStep) * pairs;
    const float back = scale[1];
    auto tiles = [&](int i, TileAt &at) {
        const int t = i * gridDim.x + blockIdx.x;
        if (t >= tiles_m * tiles_n) return false;
        place_of_tile(t, tiles_m, tiles_n, at.m, at.n);
        at.m0 = at.m * Tile::kM;
        at.n0 = at.n * Tile::kN;
        at.first = 0;
        at.last = steps;
        return true;
    };
    Tile tile;
    tile.run(hidden_t, slopes, pairs, lds, tiles, [&](const TileAt &at) {
        const int d = at.m0 + Tile::m_of();
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            const int v = at.n0 + Tile::n_of() + j;
            if (v >= tokens) continue;
            float x[Tile::kLaneM];
#pragma unroll
            for (int i = 0; i < Tile::kLaneM; ++i) x[i] = tile.acc[i / 4][j][i % 4] * back;
#pragma unroll
            for (int i = 0; i < Tile::kLaneM; i += 8) put_eight<F, false>(x + i, out + v * out_stride, d + i, dim);
        }
    });
}

template <class S>
__global__ __launch_bounds__(256) void zero_rows_kernel(S *at, int dim, int64_t stride) {
    for (int d = blockIdx.y * 256 + threadIdx.x; d < dim; d += gridDim.y * 256) at[blockIdx.x * stride + d] = 0;
}

// ------------------------------------------------------------------------------------------------- host

size_t up(size_t n, size_t to) { return (n + to - 1) / to * to; }

// Where everything lies in the workspace, and how the vocabulary is cut.
struct Plan {
    int planes, slope_planes, padded_rows, pieces, piece; // tokens of a piece: a multiple of kMostTokens
    bool packs_weight;                                   // the weights' rows are not as the products read them
    int dim_bytes, rows_bytes, piece_bytes;              // of a plane of a packed row: of hidden states and weights, and of the slopes along rows and tokens
    int form;                                            // of the tiles
    int splits, sums_stride;
    size_t count, scale, place, row, target, weight, target_logit, parts, packed_hidden, packed_weight, stats, slopes_by_row, slopes_by_token, weight_t, hidden_t, sums, bytes;
};
constexpr int kMostTokens = 256;                         // of a tile
constexpr size_t kPieceBytes = (size_t)1 << 30;
// Slopes are summed over all rows, or all tokens.  Roundings of many rows' slopes come out as one of them does, beside that of the result; of few
// rows a gradient can have one slope's, whole.  These have slopes of two parts, 16 or 22 bits: their products wait for memory in any case.
constexpr int kFewRows = 128;

// Tiles by their rows.  A vocabulary in few tiles has small ones, many steps ahead: there are more of them, and each waits for its next step less.
// us of one product, 4,096 numbers a row in bf16 (TB/s or TFLOP/s): 57,344 tokens and 32 rows in tiles of 128 x 32 86 (5.5), 256 x 32 98; 64 rows in
// 256 x 64 87 (5.4), 128 x 64 93, 64 x 64 103; 128 rows in 256 x 128 by eight waves 96 (4.9), by four 108, 128 x 128 106; 42,752 tokens and 3,840
// rows in 256 x 256 1,190 (1,130), 256 x 128 1,330 (1,010), 128 x 128 1,760, 256 x 256 by four waves 1,860.
enum Form { kFew, kRows32, kRows64, kRows128, kRows256 };
int rows_of_form(int form) { return form == kRows32 ? 32 : form == kFew || form == kRows64 ? 64 : form == kRows128 ? 128 : 256; }
template <class T, class Fn>
hipError_t with_tile(int form, Fn fn) {
    switch (form) {
        case kFew: return fn((ProductTile<T, 64, 64, 1, 2, 128, 8> *)nullptr);
        case kRows32: return fn((ProductTile<T, 128, 32, 2, 1, 128, 4> *)nullptr);
        case kRows64: return fn((ProductTile<T, 256, 64, 4, 1, 128, 3> *)nullptr);
        case kRows128: return fn((ProductTile<T, 256, 128, 4, 2, 128, 3> *)nullptr);
        default: return fn((ProductTile<T, 256, 256, 4, 2, 128, 2> *)nullptr);
    }
}
size_t tiles_of(size_t m, size_t n, int side_m, int side_n) { return (m + side_m - 1) / side_m * ((n + side_n - 1) / side_n); }
constexpr size_t kFewTiles = 128;
int form_of(int rows, int tokens) {
    if (tiles_of(tokens, rows, 256, std::min(rows, 256)) < kFewTiles) return kFew;
    if (rows <= 128) return rows <= 32 ? kRows32 : rows <= 64 ? kRows64 : kRows128;
    // (rows that fill the tiles up cost as others; 1,010 and 1,130 TFLOP/s)
    return up(rows, 128) * 1130 < up(rows, 256) * 1010 ? kRows128 : kRows256;
}

Plan plan_of(const HeadRows &h, bool grads) {
    Plan p{};
    p.planes = h.type == kLogitF32 ? 3 : 1;
    p.slope_planes = p.planes > 1 ? 3 : h.rows <= kFewRows ? 2 : 1;
    const size_t size = h.type == kLogitF32 ? 4 : 2;
    p.form = form_of(h.rows, h.vocab);
    p.padded_rows = (int)up(h.rows, std::max(rows_of_form(p.form), kStepRows));
    p.dim_bytes = (int)up((size_t)h.dim * 2, kStepBytes);
    p.packs_weight = p.planes > 1 || h.dim % 8 != 0 || (reinterpret_cast<uintptr_t>(h.weight) | (uintptr_t)(h.weight_stride * size)) % 16 != 0 || h.weight_stride >= 1 << 22;
    // what a token takes while its piece is worked on
    const size_t each = (p.packs_weight ? (size_t)p.planes * p.dim_bytes : 0) + (grads ? 2 * (2 * (size_t)p.slope_planes * p.padded_rows + p.planes * (size_t)h.dim) : 0);
    const size_t most = each ? std::max<size_t>(kMostTokens, kPieceBytes / each / kMostTokens * kMostTokens) : up(h.vocab, kMostTokens);
    p.pieces = (int)((h.vocab + most - 1) / most);
    p.piece = (int)up((h.vocab + p.pieces - 1) / p.pieces, kMostTokens);
    p.pieces = (h.vocab + p.piece - 1) / p.piece;
    p.rows_bytes = p.padded_rows * 2;
    p.piece_bytes = p.piece * 2;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t from = at; at += up(bytes, 256); return from; };
    p.count = take(4);
    p.scale = take(8);
    for (size_t *x : {&p.place, &p.row, &p.target, &p.weight, &p.target_logit}) *x = take((size_t)h.rows * 4);
    p.packed_hidden = take((size_t)p.padded_rows * p.planes * p.dim_bytes);
    p.stats = take((size_t)h.rows * 8);
    if (p.packs_weight) p.packed_weight = take(up(p.piece, kPackSide) * p.planes * p.dim_bytes);
    if (grads) {
        p.weight_t = take((size_t)h.dim * p.planes * p.piece_bytes);
        p.hidden_t = take((size_t)h.dim * p.planes * p.rows_bytes);
    }
    const size_t both = at;
    p.parts = take(up(h.vocab, kMostTokens) / kPartTokens * p.padded_rows * 8);
    if (grads) {
        const size_t forward = at;
        at = both;                                       // (the parts have been joined by then)
        p.slopes_by_row = take((size_t)p.padded_rows * p.slope_planes * p.piece_bytes);
        p.slopes_by_token = take((size_t)p.piece * p.slope_planes * p.rows_bytes);
        // few tiles of d hidden: the piece's steps are split until every unit has a tile, of at least 16 steps
        const int steps = p.piece_bytes / kStepBytes * pairs_of(p.planes, p.slope_planes);
        const int tiles = (int)tiles_of(h.dim, p.padded_rows, p.form == kFew ? 64 : p.form == kRows32 ? 128 : 256, rows_of_form(p.form));
        p.splits = std::max(1, std::min(256 / tiles, steps / 16));
        p.sums_stride = (int)up(h.dim, kLaneTokens);
        p.sums = take((size_t)p.splits * p.padded_rows * p.sums_stride * 4);
        at = std::max(at, forward);
    }
    p.bytes = at;
    return p;
}

struct Work {
    char *at;
    template <class T> T *as(size_t offset) const { return reinterpret_cast<T *>(at + offset); }
};
Taught taught_of(const Plan &p, const Work &w) {
    return {w.as<int32_t>(p.count), w.as<float>(p.scale), w.as<int32_t>(p.place), w.as<int32_t>(p.row), w.as<int32_t>(p.target), w.as<float>(p.weight)};
}

// A block takes a unit to itself, or shares it with others where they fit.
template <class Tile, class Kernel, class... Args>
hipError_t launch_tiles(Kernel kernel, int tiles, hipStream_t stream, Args... args) {
    constexpr int threads = Tile::kThreads, lds = Tile::kLdsBytes, most = kUnits * (160 * 1024 / lds);
    // (a launch may have more than 64 KiB of LDS once its kernel is told so, on every device)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(std::min(tiles, most)), dim3(threads), lds, stream, args...);
    return hipGetLastError();
}

template <class T, class F>
struct Head {
    typedef typename F::Stored Stored;
    typedef std::conditional_t<sizeof(Stored) == 4, LogitsBf16, F> Part;          // what slopes are made of
    const HeadRows &h;
    const Plan p;
    const Work w;
    const Taught taught;
    const HeadMask mask;
    hipStream_t stream;

    Head(const HeadRows &h_, bool grads, void *workspace, hipStream_t stream_)
        : h(h_), p(plan_of(h_, grads)), w{static_cast<char *>(workspace)}, taught(taught_of(p, w)), mask{h_.bitmask, h_.vocab, (h_.vocab + 31) / 32}, stream(stream_) {}

    const Stored *weight_at(int v0) const { return static_cast<const Stored *>(h.weight) + (int64_t)v0 * h.weight_stride; }
    int tokens_of(int v0) const { return std::min(p.piece, h.vocab - v0); }
    Pack pack_hidden(bool rows, bool transposed) const {
        return {h.hidden, h.hidden_stride, taught.row, taught.count, h.rows, h.dim, p.padded_rows, rows ? w.as<char>(p.packed_hidden) : nullptr,
                transposed ? w.as<char>(p.hidden_t) : nullptr, p.dim_bytes, p.rows_bytes};
    }
    Pack pack_weight(int v0, bool rows, bool transposed) const {
        const int tokens = tokens_of(v0);
        return {weight_at(v0), h.weight_stride, nullptr, nullptr, tokens, h.dim, (int)up(tokens, kPackSide), rows && p.packs_weight ? w.as<char>(p.packed_weight) : nullptr,
                transposed ? w.as<char>(p.weight_t) : nullptr, p.dim_bytes, p.piece_bytes};
    }
    Operand hidden() const { return {w.as<char>(p.packed_hidden), (int64_t)p.planes * p.dim_bytes, p.padded_rows, p.dim_bytes}; }
    Operand weight(int v0) const {
        if (!p.packs_weight) return {reinterpret_cast<const char *>(weight_at(v0)), h.weight_stride * 2, tokens_of(v0), h.dim * 2};
        return {w.as<char>(p.packed_weight), (int64_t)p.planes * p.dim_bytes, tokens_of(v0), p.dim_bytes};
    }
    int pairs() const { return pairs_of(p.planes, p.planes); }

    hipError_t stats(int v0) const {
        return with_tile<T>(p.form, [&](auto *tile) {
            typedef std::remove_pointer_t<decltype(tile)> Tile;
            const int tiles_m = (tokens_of(v0) + Tile::kM - 1) / Tile::kM;
            return launch_tiles<Tile>(head_stats_kernel<T, Tile>, tiles_m * (p.padded_rows / Tile::kN), stream, weight(v0), hidden(), pairs(), p.dim_bytes / Tile::kStep * pairs(), v0, tiles_m,
                                      mask, (const int32_t *)taught.count, (const int32_t *)taught.row, (const int32_t *)taught.target, w.as<float2>(p.parts), p.padded_rows,
                                      w.as<float>(p.target_logit));
        });
    }
    template <int kRows>
    hipError_t join(float *loss, float *stats) const {
        hipLaunchKernelGGL((head_join_kernel<kRows>), dim3((h.rows + kRows - 1) / kRows), dim3(1024), 0, stream, taught.place, h.rows, w.as<float2>(p.parts), p.padded_rows,
                           (h.vocab + kPartTokens - 1) / kPartTokens, w.as<float>(p.target_logit), loss, reinterpret_cast<float2 *>(stats));
        return hipGetLastError();
    }
    template <int kPlanes>
    hipError_t slopes(int v0, const float *stats, const Slopes &out) const {
        return with_tile<T>(p.form, [&](auto *tile) {
            typedef std::remove_pointer_t<decltype(tile)> Tile;
            const int tiles_m = (tokens_of(v0) + Tile::kM - 1) / Tile::kM;
            return launch_tiles<Tile>(head_slopes_kernel<T, Part, Tile, kPlanes>, tiles_m * (p.padded_rows / Tile::kN), stream, weight(v0), hidden(), pairs(),
                                      p.dim_bytes / Tile::kStep * pairs(), v0, tiles_m, mask, taught, reinterpret_cast<const float2 *>(stats), out);
        });
    }
    hipError_t slopes(int v0, const float *stats, const Slopes &out) const {
        if constexpr (sizeof(Stored) == 4) return slopes<3>(v0, stats, out);
        else return p.slope_planes == 2 ? slopes<2>(v0, stats, out) : slopes<1>(v0, stats, out);
    }
    hipError_t hidden_grad(int v0, const Slopes &slopes) const {
        const int pairs = pairs_of(p.planes, p.slope_planes);
        const Operand weight_t{w.as<char>(p.weight_t), (int64_t)p.planes * p.piece_bytes, h.dim, p.piece_bytes}, by_row{slopes.by_row, slopes.row_stride, p.padded_rows, p.piece_bytes};
        return with_tile<T>(p.form, [&](auto *tile) {
            typedef std::remove_pointer_t<decltype(tile)> Tile;
            const int tiles_d = (h.dim + Tile::kM - 1) / Tile::kM, steps = (tokens_of(v0) * 2 + kStepBytes - 1) / kStepBytes * pairs;
            return launch_tiles<Tile>(head_hidden_grad_kernel<T, Tile>, tiles_d * p.splits * ((p.padded_rows + Tile::kN - 1) / Tile::kN), stream, weight_t, by_row, pairs, steps, p.splits,
                                      tiles_d, (const int32_t *)taught.count, w.as<float>(p.sums), p.sums_stride, p.padded_rows, v0 == 0);
        });
    }
    hipError_t weight_grad(int v0, const Slopes &slopes, Stored *out, int64_t out_stride) const {
        const int tokens = tokens_of(v0), pairs = pairs_of(p.planes, p.slope_planes);
        const Operand hidden_t{w.as<char>(p.hidden_t), (int64_t)p.planes * p.rows_bytes, h.dim, p.rows_bytes}, by_token{slopes.by_token, slopes.token_stride, tokens, p.rows_bytes};
        return with_tile<T>(form_of(tokens, h.dim), [&](auto *tile) {
            typedef std::remove_pointer_t<decltype(tile)> Tile;
            const int tiles_d = (h.dim + Tile::kM - 1) / Tile::kM, tiles_v = (tokens + Tile::kN - 1) / Tile::kN;
            return launch_tiles<Tile>(head_weight_grad_kernel<T, F, Tile>, tiles_d * tiles_v, stream, hidden_t, by_token, pairs, tiles_d, tiles_v, (const int32_t *)taught.count,
                                      (const float *)taught.scale, h.dim, tokens, out + (int64_t)v0 * out_stride, out_stride);
        });
    }

    hipError_t run(bool forward, bool backward, float *loss, float *stats, const float *row_weight, int64_t weight_stride, Stored *grad_hidden, int64_t grad_hidden_stride,
                   Stored *grad_weight, int64_t grad_weight_stride) const {
        hipError_t e = hipSuccess;
        auto step = [&](hipError_t of) { return (e = of) == hipSuccess; };
        const bool hidden_t = backward && grad_weight, weight_t = backward && grad_hidden, whole = p.pieces == 1;
        if (!stats) stats = w.as<float>(p.stats);
        hipLaunchKernelGGL(head_rows_kernel, dim3(1), dim3(kRowsThreads), 0, stream, h.targets, h.target_bytes, h.bitmask, h.rows, h.vocab, taught, backward, row_weight, weight_stride,
                           h.type == kLogitF16);
        if (forward) {
            for (int v0 = 0; v0 < h.vocab; v0 += p.piece)           // (a vocabulary in one piece is packed once for both passes)
                if (!step(launch_pack<F>(pack_hidden(v0 == 0, v0 == 0 && hidden_t), pack_weight(v0, true, whole && weight_t), stream)) || !step(this->stats(v0))) return e;
            if (!step(h.rows <= kFewRows ? join<1>(loss, stats) : join<16>(loss, stats))) return e;
        }
        if (!backward) return hipGetLastError();
        const Slopes to{grad_hidden ? w.as<char>(p.slopes_by_row) : nullptr, grad_weight ? w.as<char>(p.slopes_by_token) : nullptr, (int64_t)p.slope_planes * p.piece_bytes,
                        (int64_t)p.slope_planes * p.rows_bytes, p.piece_bytes, p.rows_bytes};
        for (int v0 = 0; v0 < h.vocab; v0 += p.piece) {
            const bool again = !forward && v0 == 0;
            if (!(forward && whole) && !step(launch_pack<F>(pack_hidden(again, again && hidden_t), pack_weight(v0, true, weight_t), stream))) return e;
            if (!step(slopes(v0, stats, to))) return e;
            if (grad_hidden && !step(hidden_grad(v0, to))) return e;
            if (grad_weight && !step(weight_grad(v0, to, grad_weight, grad_weight_stride))) return e;
        }
        if (grad_hidden)
            hipLaunchKernelGGL((head_hidden_join_kernel<F>), dim3(h.rows, (h.dim + 1023) / 1024), dim3(256), 0, stream, taught.place, taught.scale, w.as<float>(p.sums), p.splits,
                               p.sums_stride, p.padded_rows, h.dim, grad_hidden, grad_hidden_stride);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_zero_rows(void *at, LogitType type, int rows, int dim, int64_t stride, hipStream_t stream) {
    const dim3 grid(rows, (dim + 1023) / 1024);
    if (type == kLogitF32) hipLaunchKernelGGL((zero_rows_kernel<uint32_t>), grid, dim3(256), 0, stream, static_cast<uint32_t *>(at), dim, stride);
    else hipLaunchKernelGGL((zero_rows_kernel<uint16_t>), grid, dim3(256), 0, stream, static_cast<uint16_t *>(at), dim, stride);
    return hipGetLastError();
}

size_t head_workspace_bytes(const HeadRows &h, bool grads) { return plan_of(h, grads).bytes; }

hipError_t launch_head(const HeadRows &h, bool forward, bool backward, float *loss, float *stats, const float *row_weight, int64_t weight_stride, void *grad_hidden,
                       int64_t grad_hidden_stride, void *grad_weight, int64_t grad_weight_stride, void *workspace, hipStream_t stream) {
    auto run = [&](const auto &head) {
        typedef typename std::decay_t<decltype(head)>::Stored Stored;
        return head.run(forward, backward, loss, stats, row_weight, weight_stride, static_cast<Stored *>(grad_hidden), grad_hidden_stride, static_cast<Stored *>(grad_weight), grad_weight_stride);
    };
    switch (h.type) {
        case kLogitBf16: return run(Head<ProductBf16, LogitsBf16>(h, backward, workspace, stream));
        case kLogitF16: return run(Head<ProductF16, LogitsF16>(h, backward, workspace, stream));
        default: return run(Head<ProductBf16, LogitsF32>(h, backward, workspace, stream));
    }
}

}  // namespace pre3
