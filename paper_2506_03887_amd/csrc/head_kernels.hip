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
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, words = (vocab + 31) / 32;
    int before = 0;
    float top = 0.0f;
    for (int r0 = 0; r0 < rows; r0 += kRowsThreads) {
        const int r = r0 + tid;
        int target = -1;
        if (r < rows) {
            const int64_t t = id_at(targets, target_bytes, r);
            if (t >= 0 && t < vocab && (!bitmask || (bitmask[(size_t)r * words + (t >> 5)] >> (t & 31) & 1u))) target = (int)t;
        }
        const bool is = target >= 0;
        const uint64_t them = __ballot(is);
        if (lane == 0) sums[wave] = __popcll(them);
        __syncthreads();
        int at = before + __popcll(them & ((1ull << lane) - 1));
        for (int w = 0; w < kRowsThreads / 64; ++w) {
            if (w < wave) at += sums[w];
            before += sums[w];
        }
        __syncthreads();
        if (r < rows) taught.place[r] = is ? at : -1;
        if (is) {
            taught.row[at] = r;
            taught.target[at] = target;
            if (weighted) {
                const float g = row_weight ? row_weight[(int64_t)r * weight_stride] : 1.0f;
                taught.weight[at] = g;
                if (fabsf(g) < INFINITY) top = fmaxf(top, fabsf(g));
            }
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
// The tiles of a block over the taught rows (in whole steps of kStepRows) and a piece's tokens.
constexpr int kStepRows = kStepBytes / 2;
template <class Tile>
struct RowTiles {
    int tiles_m, tiles_n, steps;
    __device__ RowTiles(int tiles_m_, int rows, int steps_) : tiles_m(tiles_m_), tiles_n(((rows + kStepRows - 1) / kStepRows * kStepRows + Tile::kN - 1) / Tile::kN), steps(steps_) {}
    __device__ bool operator()(int i, TileAt &at) const {
        const int tile = i * gridDim.x + blockIdx.x;
        if (tile >= tiles_m * tiles_n) return false;
        place_of_tile(tile, tiles_m, tiles_n, at.m, at.n);
        at.m0 = at.m * Tile::kM;
        at.n0 = at.n * Tile::kN;
        at.first = 0;
        at.last = steps;
        return true;
    }
};

// Maximum, and sum of the exponentials over it, of every taught row over a wave's share of a tile's tokens; a target's logit.
template <class T, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head_stats_kernel(Operand weight, Operand hidden, int pairs, int steps, int v0, int tiles_m, HeadMask mask, const int32_t *count,
                                                                    const int32_t *row_of, const int32_t *target_of, float2 *parts, int parts_stride, float *target_logit) {
    static_assert(Tile::kLaneM == kLaneTokens, "a lane's tokens");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int rows = *count;
    Tile tile;
    tile.run(weight, hidden, pairs, lds, RowTiles<Tile>(tiles_m, rows, steps), [&](const TileAt &at) {
        const int v = v0 + at.m0 + Tile::m_of(), first = at.n0 + Tile::n_of();
        float2 *out = parts + (size_t)((v0 / Tile::kM + at.m) * Tile::kWavesM + Tile::wave() / Tile::kWavesN) * parts_stride;
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

// A row's parts joined, kRows rows to a block: of the largest maximum, and the sums in 64 bits.
template <int kRows>
__global__ __launch_bounds__(256) void head_join_kernel(const int32_t *place, int rows, const float2 *parts, int parts_stride, int n_parts, const float *target_logit, float *loss,
                                                        float2 *stats) {
    constexpr int kOver = 256 / kRows;                                    // threads of a row
    __shared__ float tops[kOver][kRows];
    __shared__ double sums[kOver][kRows];
    const int i = threadIdx.x % kRows, part = threadIdx.x / kRows, r = blockIdx.x * kRows + i;
    const int at = r < rows ? place[r] : -1;
    float top = -INFINITY;
    if (at >= 0)
        for (int p = part; p < n_parts; p += kOver) top = fmaxf(top, parts[(size_t)p * parts_stride + at].x);
    tops[part][i] = top;
    __syncthreads();
    for (int p = 0; p < kOver; ++p) top = fmaxf(top, tops[p][i]);
    double sum = 0.0;
    if (at >= 0)
        for (int p = part; p < n_parts; p += kOver) {
            const float2 x = parts[(size_t)p * parts_stride + at];
            if (x.x > -INFINITY || x.y != x.y) sum += (double)(x.y * __builtin_amdgcn_exp2f((x.x - top) * kLog2E));
        }
    sums[part][i] = sum;
    __syncthreads();
    if (part || r >= rows) return;
    for (int p = 1; p < kOver; ++p) sum += sums[p][i];
    if (loss) loss[r] = at < 0 ? 0.0f : (float)(log(sum) + ((double)top - (double)target_logit[at]));
    if (stats) stats[r] = at < 0 ? make_float2(0.0f, 1.0f) : make_float2(top, (float)sum);
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
    static_assert(Tile::kLaneM == kLaneTokens, "a lane's tokens");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int rows = *taught.count;
    const float scale = taught.scale[0];
    Tile tile;
    tile.run(weight, hidden, pairs, lds, RowTiles<Tile>(tiles_m, rows, steps), [&](const TileAt &at) {
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
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j)
#pragma unroll
            for (int i = 0; i < Tile::kMi; ++i) {
                if (d + 4 * i >= sums_stride) continue;                   // (a multiple of four)
                Float4 *to = reinterpret_cast<Float4 *>(out + (size_t)j * sums_stride + 4 * i);
                *to = first ? tile.acc[i][j] : *to + tile.acc[i][j];
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
    int planes, slope_planes, padded_rows, pieces, piece; // tokens of a piece: a multiple of 256
    bool packs_weight;                                   // the weights' rows are not as the products read them
    int hidden_bytes;                                    // of a packed row's plane
    int n_tile;                                          // rows of a tile
    int splits, sums_stride;
    size_t count, scale, place, row, target, weight, target_logit, parts, packed_hidden, packed_weight, stats, slopes_by_row, slopes_by_token, weight_t, hidden_t, sums, bytes;
};
// Slopes are summed over all rows, or all tokens.  Roundings of many rows' slopes come out as one of them does, beside that of the result; of few
// rows a gradient can have one slope's, whole.  These have slopes of two parts, 16 or 22 bits: their products wait for memory in any case.
constexpr int kFewRows = 128;
// A tile has 256 tokens in every form.
constexpr int kTileTokens = 256, kWavesOfTokens = 4;
constexpr size_t kPieceBytes = (size_t)1 << 30;

int tile_rows(int rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }

Plan plan_of(const HeadRows &h, bool grads) {
    Plan p{};
    p.planes = h.type == kLogitF32 ? 3 : 1;
    const size_t size = h.type == kLogitF32 ? 4 : 2;
    p.n_tile = tile_rows(h.rows);
    p.slope_planes = p.planes > 1 ? 3 : h.rows <= kFewRows ? 2 : 1;
    p.padded_rows = (int)up(h.rows, std::max(p.n_tile, kStepRows));
    p.hidden_bytes = (int)up((size_t)h.dim * 2, kStepBytes);
    p.packs_weight = p.planes > 1 || h.dim % 8 != 0 || (reinterpret_cast<uintptr_t>(h.weight) | (uintptr_t)(h.weight_stride * size)) % 16 != 0 || h.weight_stride >= 1 << 22;
    // what a token takes while its piece is worked on
    const size_t each = (p.packs_weight ? (size_t)p.planes * p.hidden_bytes : 0) + (grads ? 2 * (2 * (size_t)p.slope_planes * p.padded_rows + p.planes * (size_t)h.dim) : 0);
    const size_t most = each ? std::max<size_t>(kTileTokens, kPieceBytes / each / kTileTokens * kTileTokens) : up(h.vocab, kTileTokens);
    p.pieces = (int)((h.vocab + most - 1) / most);
    p.piece = (int)up((h.vocab + p.pieces - 1) / p.pieces, kTileTokens);
    p.pieces = (h.vocab + p.piece - 1) / p.piece;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t from = at; at += up(bytes, 256); return from; };
    p.count = take(4);
    p.scale = take(8);
    for (size_t *x : {&p.place, &p.row, &p.target, &p.weight, &p.target_logit}) *x = take((size_t)h.rows * 4);
    p.packed_hidden = take((size_t)p.padded_rows * p.planes * p.hidden_bytes);
    p.stats = take((size_t)h.rows * 8);
    if (p.packs_weight) p.packed_weight = take((size_t)p.piece * p.planes * p.hidden_bytes);
    const size_t both = at;
    p.parts = take(up(h.vocab, kTileTokens) / kTileTokens * kWavesOfTokens * p.padded_rows * 8);
    if (grads) {
        size_t forward = at;
        at = both;                                       // (the parts have been joined by then)
        p.slopes_by_row = take((size_t)p.padded_rows * p.slope_planes * p.piece * 2);
        p.slopes_by_token = take((size_t)p.piece * p.slope_planes * p.padded_rows * 2);
        p.weight_t = take((size_t)h.dim * p.planes * p.piece * 2);
        p.hidden_t = take((size_t)h.dim * p.planes * p.padded_rows * 2);
        // few tiles of d hidden: the piece's steps are split until every unit has a tile, of at least 16 steps
        const int tiles = (int)(up(h.dim, kTileTokens) / kTileTokens * (p.padded_rows / p.n_tile)), steps = p.piece * 2 / kStepBytes * pairs_of(p.planes, p.slope_planes);
        p.splits = std::max(1, std::min(256 / tiles, steps / 16));
        p.sums_stride = (int)up(h.dim, 4);
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

// A block takes a unit to itself, or shares it with another where two fit.
template <class Tile, class Kernel, class... Args>
hipError_t launch_tiles(Kernel kernel, int tiles, hipStream_t stream, Args... args) {
    constexpr int threads = Tile::kThreads, lds = Tile::kLdsBytes, most = kUnits * (160 * 1024 / lds);
    const int blocks = std::min(tiles, most);
    // (a launch may have more than 64 KiB of LDS once its kernel is told so, on every device)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), lds, stream, args...);
    return hipGetLastError();
}
// A tile's steps over as much of k as so many of the longest.
template <class Tile>
int steps_of(int longest) { return longest * (kStepBytes / Tile::kStep); }
// fn(a tile's type) for tiles of so many rows.
template <class T, class Fn>
hipError_t with_tile(int n_tile, Fn fn) {
    switch (n_tile) {
        case 32: return fn((ProductTile<T, 256, 32, 4, 1, 128, 4> *)nullptr);
        case 64: return fn((ProductTile<T, 256, 64, 4, 1, 128, 3> *)nullptr);
        case 128: return fn((ProductTile<T, 256, 128, 4, 1, 128, 3> *)nullptr);
        default: return fn((ProductTile<T, 256, 256, 4, 2, 128, 2> *)nullptr);
    }
}

template <class F>
Operand weight_operand(const HeadRows &h, const Plan &p, const Work &w, int v0, hipStream_t stream, hipError_t &e) {
    const int tokens = std::min(p.piece, h.vocab - v0);
    const auto *from = static_cast<const typename F::Stored *>(h.weight) + (int64_t)v0 * h.weight_stride;
    if (!p.packs_weight) return {reinterpret_cast<const char *>(from), h.weight_stride * 2, tokens, h.dim * 2};
    e = launch_pack<F>(from, h.weight_stride, nullptr, nullptr, tokens, tokens, h.dim, w.as<char>(p.packed_weight), p.hidden_bytes, stream);
    return {w.as<char>(p.packed_weight), (int64_t)p.planes * p.hidden_bytes, tokens, p.hidden_bytes};
}

template <class T, class F>
hipError_t run(const HeadRows &h, bool forward, bool backward, float *loss, float *stats, const float *row_weight, int64_t weight_stride, void *grad_hidden,
               int64_t grad_hidden_stride, void *grad_weight, int64_t grad_weight_stride, void *workspace, hipStream_t stream) {
    typedef typename F::Stored Stored;
    const Plan p = plan_of(h, backward);
    const Work w{static_cast<char *>(workspace)};
    const Taught taught = taught_of(p, w);
    const HeadMask mask{h.bitmask, h.vocab, (h.vocab + 31) / 32};
    hipError_t e = hipSuccess;
    hipLaunchKernelGGL(head_rows_kernel, dim3(1), dim3(kRowsThreads), 0, stream, h.targets, h.target_bytes, h.bitmask, h.rows, h.vocab, taught, backward, row_weight, weight_stride,
                       h.type == kLogitF16);
    const auto *hidden_rows = static_cast<const Stored *>(h.hidden);
    e = launch_pack<F>(hidden_rows, h.hidden_stride, taught.row, taught.count, h.rows, p.padded_rows, h.dim, w.as<char>(p.packed_hidden), p.hidden_bytes, stream);
    if (e != hipSuccess) return e;
    const Operand hidden{w.as<char>(p.packed_hidden), (int64_t)p.planes * p.hidden_bytes, p.padded_rows, p.hidden_bytes};
    const int pairs = pairs_of(p.planes, p.planes), steps = p.hidden_bytes / kStepBytes * pairs, tiles_n = p.padded_rows / p.n_tile;
    if (!stats) stats = w.as<float>(p.stats);
    if (forward) {
        for (int v0 = 0; v0 < h.vocab; v0 += p.piece) {
            const Operand weight = weight_operand<F>(h, p, w, v0, stream, e);
            if (e != hipSuccess) return e;
            const int tiles_m = (weight.rows + kTileTokens - 1) / kTileTokens;
            e = with_tile<T>(p.n_tile, [&](auto *tile) {
                typedef std::remove_pointer_t<decltype(tile)> Tile;
                static_assert(Tile::kM == kTileTokens && Tile::kWavesM == kWavesOfTokens, "parts of a row");
                return launch_tiles<Tile>(head_stats_kernel<T, Tile>, tiles_m * tiles_n, stream, weight, hidden, pairs, steps_of<Tile>(steps), v0, tiles_m, mask, (const int32_t *)taught.count,
                                          (const int32_t *)taught.row, (const int32_t *)taught.target, w.as<float2>(p.parts), p.padded_rows, w.as<float>(p.target_logit));
            });
            if (e != hipSuccess) return e;
        }
        const int n_parts = (h.vocab + kTileTokens - 1) / kTileTokens * kWavesOfTokens;
        auto join = [&](auto rows_of_block) {
            constexpr int kRows = decltype(rows_of_block)::value;
            hipLaunchKernelGGL((head_join_kernel<kRows>), dim3((h.rows + kRows - 1) / kRows), dim3(256), 0, stream, taught.place, h.rows, w.as<float2>(p.parts), p.padded_rows, n_parts,
                               w.as<float>(p.target_logit), loss, reinterpret_cast<float2 *>(stats));
        };
        if (h.rows <= kFewRows) join(std::integral_constant<int, 1>());
        else join(std::integral_constant<int, 16>());
    }
    if (!backward) return hipGetLastError();
    const int rows_bytes = p.padded_rows * 2, piece_bytes = p.piece * 2, slope_pairs = pairs_of(p.planes, p.slope_planes);
    if (grad_weight) {
        e = launch_pack_transposed<F>(hidden_rows, h.hidden_stride, taught.row, taught.count, h.rows, p.padded_rows, h.dim, w.as<char>(p.hidden_t), rows_bytes, stream);
        if (e != hipSuccess) return e;
    }
    const Slopes slopes{grad_hidden ? w.as<char>(p.slopes_by_row) : nullptr, grad_weight ? w.as<char>(p.slopes_by_token) : nullptr, (int64_t)p.slope_planes * piece_bytes,
                        (int64_t)p.slope_planes * rows_bytes, piece_bytes, rows_bytes};
    for (int v0 = 0; v0 < h.vocab; v0 += p.piece) {
        const Operand weight = weight_operand<F>(h, p, w, v0, stream, e);
        if (e != hipSuccess) return e;
        const int tokens = weight.rows, tiles_m = (tokens + kTileTokens - 1) / kTileTokens, tiles_d = (h.dim + kTileTokens - 1) / kTileTokens;
        e = with_tile<T>(p.n_tile, [&](auto *tile) {
            typedef std::remove_pointer_t<decltype(tile)> Tile;
            // (tiles of few rows have slopes of two parts, those of many have one)
            constexpr int kPlanes = sizeof(Stored) == 4 ? 3 : Tile::kN <= kFewRows ? 2 : 1;
            return launch_tiles<Tile>(head_slopes_kernel<T, std::conditional_t<sizeof(Stored) == 4, LogitsBf16, F>, Tile, kPlanes>, tiles_m * tiles_n, stream, weight, hidden, pairs,
                                      steps_of<Tile>(steps), v0, tiles_m, mask, taught, reinterpret_cast<const float2 *>(stats), slopes);
        });
        if (e != hipSuccess) return e;
        if (grad_hidden) {
            const auto *from = static_cast<const Stored *>(h.weight) + (int64_t)v0 * h.weight_stride;
            e = launch_pack_transposed<F>(from, h.weight_stride, nullptr, nullptr, tokens, tiles_m * kTileTokens, h.dim, w.as<char>(p.weight_t), piece_bytes, stream);
            if (e != hipSuccess) return e;
            const Operand weight_t{w.as<char>(p.weight_t), (int64_t)p.planes * piece_bytes, h.dim, piece_bytes}, by_row{slopes.by_row, slopes.row_stride, p.padded_rows, piece_bytes};
            e = with_tile<T>(p.n_tile, [&](auto *tile) {
                typedef std::remove_pointer_t<decltype(tile)> Tile;
                return launch_tiles<Tile>(head_hidden_grad_kernel<T, Tile>, tiles_d * p.splits * tiles_n, stream, weight_t, by_row, slope_pairs,
                                          tiles_m * kTileTokens * 2 / kStepBytes * slope_pairs, p.splits, tiles_d, (const int32_t *)taught.count, w.as<float>(p.sums), p.sums_stride,
                                          p.padded_rows, v0 == 0);
            });
            if (e != hipSuccess) return e;
        }
        if (grad_weight) {
            const Operand hidden_t{w.as<char>(p.hidden_t), (int64_t)p.planes * rows_bytes, h.dim, rows_bytes},
                by_token{slopes.by_token, slopes.token_stride, tiles_m * kTileTokens, rows_bytes};
            typedef ProductTile<T, 256, 256, 4, 2, 128, 2> Tile;
            e = launch_tiles<Tile>(head_weight_grad_kernel<T, F, Tile>, tiles_d * tiles_m, stream, hidden_t, by_token, slope_pairs, tiles_d, tiles_m, (const int32_t *)taught.count,
                                   (const float *)taught.scale, h.dim, tokens, static_cast<Stored *>(grad_weight) + (int64_t)v0 * grad_weight_stride, grad_weight_stride);
            if (e != hipSuccess) return e;
        }
    }
    if (grad_hidden)
        hipLaunchKernelGGL((head_hidden_join_kernel<F>), dim3(h.rows, (h.dim + 1023) / 1024), dim3(256), 0, stream, taught.place, taught.scale, w.as<float>(p.sums), p.splits, p.sums_stride,
                           p.padded_rows, h.dim, static_cast<Stored *>(grad_hidden), grad_hidden_stride);
    return hipGetLastError();
}

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
    switch (h.type) {
        case kLogitBf16: return run<ProductBf16, LogitsBf16>(h, forward, backward, loss, stats, row_weight, weight_stride, grad_hidden, grad_hidden_stride, grad_weight, grad_weight_stride, workspace, stream);
        case kLogitF16: return run<ProductF16, LogitsF16>(h, forward, backward, loss, stats, row_weight, weight_stride, grad_hidden, grad_hidden_stride, grad_weight, grad_weight_stride, workspace, stream);
        default: return run<ProductBf16, LogitsF32>(h, forward, backward, loss, stats, row_weight, weight_stride, grad_hidden, grad_hidden_stride, grad_weight, grad_weight_stride, workspace, stream);
    }
}

}  // namespace pre3
