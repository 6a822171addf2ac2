// gfx950 kernels of a head's cross entropy: the loss of one target token a row in the logits  x = hidden weight^T  behind the token mask, and
// its gradients.  With p = softmax(x) over a row's allowed tokens, t its target and g the gradient of what is minimised with respect to
// its loss,
//     loss = log(sum of exp x) - x_t,      s_v = g (p_v - [v = t]),      d hidden = s weight,      d weight = s^T hidden.
// A row without a target, or whose target the mask leaves out, has no loss and no gradient: such rows are not computed at all, the others
// lie side by side in what the products read.
//
// There are three ways through, by the number of rows:
//   2 to 8         (by type) vector instructions in 32 bits: the weights are read once for the logits and once for both gradients, whatever the products take.
//   at most 128,   products in matrix instructions, split along k until every unit has a share, whose sums in 32 bits are added up by the kernel that
//   or few tiles   takes a row's maximum and sum of exponentials; the logits live as long as the call and are few beside the weights.  What bounds it is
//                  the reading of the weights: once for the loss (4.9 TB/s), and once for d hidden; d weight is written once.
//   others         the logits are never kept.  The forward pass leaves of a tile of logits its rows' maxima and sums of exponentials; the backward pass
//                  makes the logits again, writes their slopes s, and multiplies them into both gradients: four products of 2 rows x vocabulary x dim
//                  operations each, where keeping the logits would take three, and 2 to 4 bytes for every logit, several times over.  What
//                  bounds it is the rate of the products: 3,700 rows that teach, of 128,256 tokens and 4,096 numbers in bf16, take 13.9 ms, 1,120 TFLOP/s.
// Both gradients' products sum over what the operands' rows are numbered by (tokens, or rows), so they take these in columns, as they lie.
//
// Slopes are rounded to the operands' type: bf16 to 2^-8 of themselves at most, as the gradients they make are rounded after that; f16, whose range would
// lose the small ones, after a common power of two that brings the largest weight of a row to 2^14.  (Of at most 128 rows they are sums of two
// such numbers, and where vector instructions multiply them of 32 bits.)  Sums are held in 32 bits.  32-bit operands and slopes are the sums of three bf16 numbers, of 8 bits each,
// and a product of two is the six products of parts that reach its 24 bits (2 x 6 operations instead of 2, at 16 times the rate of 32-bit
// matrix instructions).
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
    int32_t *infinite;             // [1]: 1 if one of their logits, masked ones as well, is not finite
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
    if (tid == 0) { *taught.count = before; *taught.infinite = 0; }
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
__global__ __launch_bounds__(Tile::kThreads) void head_stats_kernel(Operand weight, Operand hidden, int pairs, int k_steps, int v0, int tiles_m, HeadMask mask, const int32_t *count,
                                                                    const int32_t *row_of, const int32_t *target_of, float2 *parts, int parts_stride, float *target_logit) {
    static_assert(Tile::kLaneM == kLaneTokens && Tile::kM / Tile::kWavesM == kPartTokens, "a lane's tokens");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int rows = *count;
    Tile tile;
    tile.run(weight, hidden, pairs, k_steps, lds, RowTiles<Tile, false>(tiles_m, rows, k_steps * pairs), [&](const TileAt &at) {
        const int v = v0 + at.m0 + Tile::m_of(0), first = at.n0 + Tile::n_of(0);
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

// A row's parts joined, kJoinRows rows to a block, in one pass: the sums, over the largest maximum so far, in 64 bits.
struct Joined { float top; double sum; };
__device__ __forceinline__ Joined join(Joined a, float top, double sum) {
    const float most = fmaxf(a.top, top);
    if (most == -INFINITY) return {most, a.sum + sum};                    // (nothing yet, or a NaN)
    return {most, a.sum * __builtin_amdgcn_exp2f((a.top - most) * kLog2E) + sum * __builtin_amdgcn_exp2f((top - most) * kLog2E)};
}
// What comes out of a row.
__device__ __forceinline__ void put_row(int r, bool taught, const Joined &all, float target, float *loss, float2 *stats) {
    if (loss) loss[r] = taught ? (float)(log(all.sum) + ((double)all.top - (double)target)) : 0.0f;
    if (stats) stats[r] = taught ? make_float2(all.top, (float)all.sum) : make_float2(0.0f, 1.0f);
}
constexpr int kJoinRows = 16;
__global__ __launch_bounds__(1024) void head_join_kernel(const int32_t *place, int rows, const float2 *parts, int parts_stride, int n_parts, const float *target_logit, float *loss,
                                                         float2 *stats) {
    constexpr int kRows = kJoinRows, kOver = 1024 / kRows;                // threads of a row
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
    put_row(r, at >= 0, joined[0][i], at >= 0 ? target_logit[at] : 0.0f, loss, stats);
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

// The slopes of a piece of the vocabulary, as numbers of 16 bits in one to three planes, along the tokens: zeros behind the last token and from the last taught
// row to the end of its step.
struct Slopes {
    char *at;
    int64_t row_stride, plane;
};
template <class T, class F, class Tile, int kPlanes>
__global__ __launch_bounds__(Tile::kThreads) void head_slopes_kernel(Operand weight, Operand hidden, int pairs, int k_steps, int v0, int tiles_m, HeadMask mask, Taught taught,
                                                                     const float2 *stats, Slopes out) {
    static_assert(Tile::kLaneM == kLaneTokens && Tile::kM / Tile::kWavesM == kPartTokens, "a lane's tokens");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int rows = *taught.count;
    const float scale = taught.scale[0];
    Tile tile;
    tile.run(weight, hidden, pairs, k_steps, lds, RowTiles<Tile, true>(tiles_m, rows, k_steps * pairs), [&](const TileAt &at) {
        const int m = at.m0 + Tile::m_of(0), v = v0 + m, first = at.n0 + Tile::n_of(0);
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
        float zero[Tile::kNj];                                            // (0 as long as all are finite)
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            zero[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < kLaneTokens; ++i) zero[j] = fmaf(tile.acc[i / 4][j][i % 4], 0.0f, zero[j]);
            if (zero[j] != 0.0f) *taught.infinite = 1;
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
#pragma unroll
            for (int j = 0; j < Tile::kNj; ++j) {
                float x[kLaneTokens];
#pragma unroll
                for (int i = 0; i < kLaneTokens; ++i) x[i] = tile.acc[i / 4][j][i % 4];
                put_16_bit<F, kLaneTokens>(x, out.at + (first + j) * out.row_stride + plane * out.plane + m * 2);
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

// How many shares the sums of d hidden have: of those that there is room for, as many as give every block of the launch a tile.
__device__ __forceinline__ int shares_of(int tiles_m, int tile_n, int rows, int blocks, int most) {
    const int tiles = tiles_m * ((rows + tile_n - 1) / tile_n);
    return max(1, min(most, blocks / max(tiles, 1)));
}
struct Shares { int tiles_m, tile_n, blocks, most; };

// A product with slopes: a masked token's is zero, and stays it whatever the token's weights or the row's hidden states are.  If there are some that are not
// finite then a logit is not either, and only then are the operands cleared of them: that takes 8 % of a product of 2,048 rows.
template <class Tile, class Tiles, class Done>
__device__ __forceinline__ void run_finite(Tile &tile, const int32_t *infinite, const Operand &a, const Operand &b, int pairs, int k_steps, char *lds, Tiles tiles, Done done) {
    if constexpr (Tile::kColumnsA)
        if (*infinite) return tile.template run<true>(a, b, pairs, k_steps, lds, tiles, done);
    tile.run(a, b, pairs, k_steps, lds, tiles, done);
}

// Sums of a product in 32 bits, [split][n][m], of which each split takes its share of the steps: d hidden over a piece of the vocabulary, added to that of
// the pieces before (first: there is none), the logits of few rows, and d weight of few tokens.  rows: n's that there are (null: all of b's).  along: rows that the
// steps go through (null: k_steps).  fitted: as many shares as the rows leave blocks for, at most `splits`; else as many as that.
template <class T, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head_sums_kernel(Operand a, Operand b, int pairs, int k_steps, int splits, int tiles_m, const int32_t *rows, const int32_t *along, const int32_t *infinite, float *sums,
                                                                   int64_t sums_stride, int64_t split_stride, int sums_m, int n_all, bool first, bool fitted) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    static_assert(Tile::kLaneM == kLaneTokens, "a lane's numbers");
    if (along) k_steps = (*along + kStepRows - 1) / kStepRows;
    const int there = rows ? *rows : n_all, tiles_n = (there + Tile::kN - 1) / Tile::kN, steps = k_steps * pairs;       // (of no rows: none, and sums of zero)
    if (fitted) splits = shares_of(tiles_m, Tile::kN, there, gridDim.x, splits);
    auto tiles = [&](int i, TileAt &at) {
        const int t = i * gridDim.x + blockIdx.x;
        if (t >= tiles_m * splits * tiles_n) return false;
        place_of_tile(t, tiles_m * splits, tiles_n, at.m, at.n);
        const int split = at.m / tiles_m;
        at.m0 = (at.m - split * tiles_m) * Tile::kM;
        at.n0 = at.n * Tile::kN;
        at.first = steps * split / splits;
        at.last = steps * (split + 1) / splits;
        return true;
    };
    Tile tile;
    run_finite(tile, infinite, a, b, pairs, max(k_steps, 1), lds, tiles, [&](const TileAt &at) {
        float *out = sums + (at.m / tiles_m) * split_stride;
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            const int n = at.n0 + Tile::n_of(j);
            if (n >= there) continue;
            auto place = [&](int i) { return reinterpret_cast<Float4 *>(out + n * sums_stride + at.m0 + Tile::m_of(i)); };
            Float4 sum[Tile::kMi];
#pragma unroll
            for (int i = 0; i < Tile::kMi; ++i) sum[i] = first || at.m0 + Tile::m_of(i) >= sums_m ? Float4{0, 0, 0, 0} : *place(i);
#pragma unroll
            for (int i = 0; i < Tile::kMi; ++i)
                if (at.m0 + Tile::m_of(i) < sums_m) *place(i) = sum[i] + tile.acc[i][j];
        }
    });
}

// ---- few rows, or a vocabulary in few tiles: the logits are sums in 32 bits that live as long as the call, far fewer than the weights, and the products are
// split along k until every unit has a share.

// A stretch of a row for every block: the splits' sums added up (and left in `kept`), maximum and sum of exponentials, the target's logit.  Where a row is one
// stretch, its loss and stats as well (parts null).
constexpr int kRowThreads = 512, kRowTokens = 4 * 4 * kRowThreads;
__global__ __launch_bounds__(kRowThreads) void head_row_kernel(const int32_t *place, HeadMask mask, const int32_t *target_of, const float *logits, int64_t stride, int64_t split_stride, int splits,
                                                               float *kept, int tokens_of_block, float2 *parts, int parts_stride, float *target_logit, float *loss, float2 *stats) {
    __shared__ Joined joined[kRowThreads / 64];
    __shared__ float of_target;
    const int r = blockIdx.x, tid = threadIdx.x, at = place[r];
    if (at < 0) {
        if (!parts && tid == 0) put_row(r, false, Joined{}, 0.0f, loss, stats);
        return;
    }
    const int begin = blockIdx.y * tokens_of_block, end = min(mask.vocab, begin + tokens_of_block);
    const int target = target_of[at];
    const uint32_t *bits = mask.bitmask ? mask.bitmask + (size_t)r * mask.words : nullptr;
    constexpr int kAhead = 4, kOver = 4 * kRowThreads;                    // groups of four tokens on their way, tokens of a round of the block
    float top = -INFINITY, sum = 0.0f;
    for (int v0 = begin + tid * 4; v0 < end; v0 += kAhead * kOver) {
        Float4 x[kAhead];
        uint32_t allowed[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int v = v0 + i * kOver, left = end - v;
            allowed[i] = left <= 0 ? 0u : left >= 4 ? 0xFu : (1u << left) - 1u;
            if (left > 0) x[i] = *reinterpret_cast<const Float4 *>(logits + at * stride + v);
            if (left > 0 && bits) allowed[i] &= bits[v >> 5] >> (v & 31);
        }
        if (splits > 1) {
            for (int s = 1; s < splits; ++s)
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (v0 + i * kOver < end) x[i] += *reinterpret_cast<const Float4 *>(logits + s * split_stride + at * stride + v0 + i * kOver);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (v0 + i * kOver < end) *reinterpret_cast<Float4 *>(kept + at * stride + v0 + i * kOver) = x[i];
        }
        float most = top;
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (v0 + i * kOver + e == target) of_target = x[i][e];
                x[i][e] = allowed[i] >> e & 1u ? x[i][e] : -INFINITY;
                most = fmaxf(most, x[i][e]);
            }
        const float base = most == -INFINITY ? 0.0f : most;
        sum *= __builtin_amdgcn_exp2f((top - base) * kLog2E);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((x[i][e] - base) * kLog2E);
        top = most;
    }
    Joined all = {top, sum};
#pragma unroll
    for (int apart = 32; apart > 0; apart /= 2) all = join(all, __shfl_xor(all.top, apart), __shfl_xor(all.sum, apart));
    if (tid % 64 == 0) joined[tid / 64] = all;
    __syncthreads();
    if (tid) return;
    for (int w = 1; w < kRowThreads / 64; ++w) all = join(all, joined[w].top, joined[w].sum);
    if (!parts) return put_row(r, true, all, of_target, loss, stats);
    parts[(size_t)blockIdx.y * parts_stride + at] = make_float2(all.top, (float)all.sum);
    if (target >= begin && target < end) target_logit[at] = of_target;
}

// The slopes of 64 rows and 64 tokens of a piece out of their logits (rows of the whole vocabulary's), four by four a thread.
template <class F, int kPlanes>
__global__ __launch_bounds__(256) void head_row_slopes_kernel(const float *logits, int64_t stride, int v0, HeadMask mask, Taught taught, const float2 *stats, int row_limit, Slopes out) {
    const int rows = *taught.count, m = blockIdx.x * 64 + threadIdx.x % 16 * 4, v = v0 + m, first = blockIdx.y * 64 + threadIdx.x / 16 * 4;
    const float scale = taught.scale[0];
    float x[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = first + j;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[j][e] = 0.0f;
        if (n >= rows || v >= mask.vocab) continue;
        const int row = taught.row[n], target = taught.target[n] - v;
        const float2 sum = stats[row];
        const float g = taught.weight[n] * scale, share = 1.0f / sum.y;
        uint32_t allowed = mask.vocab - v >= 4 ? 0xFu : (1u << (mask.vocab - v)) - 1u;
        if (mask.bitmask) allowed &= mask.bitmask[(size_t)row * mask.words + (v >> 5)] >> (v & 31);
        const Float4 logit = *reinterpret_cast<const Float4 *>(logits + n * stride + v);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (v + e < mask.vocab && !(fabsf(logit[e]) < INFINITY)) *taught.infinite = 1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float p = __builtin_amdgcn_exp2f((logit[e] - sum.x) * kLog2E) * share;
            if (target == e) p -= 1.0f;
            x[j][e] = allowed >> e & 1u ? p * g : 0.0f;
        }
    }
#pragma unroll
    for (int plane = 0; plane < kPlanes; ++plane) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (first + j < row_limit) put_16_bit<F, 4>(x[j], out.at + (first + j) * out.row_stride + plane * out.plane + m * 2);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][e] -= F::value(F::pattern(x[j][e]));
    }
}

// The logits of few rows from weights that do not lie as a tile fetches them (odd strides, 32 bits): a lane reads its share of a matrix instruction's operand from
// memory, eight numbers of a token's row, and takes it apart itself; packing them first writes and reads them once more (32 bits: reads the six
// products' parts, 12 bytes a number instead of 4).  Of a loss alone: a backward pass has packed weights in any case.  A wave has 64 tokens and kN rows; of 32-bit numbers the largest parts' product has sums of its own,
// as the others', up to 2^-8 of its size, would otherwise round it six times as often.
template <class T, class F, int kN>
__global__ __launch_bounds__(256) void head_direct_kernel(const typename F::Stored *weight, int64_t weight_stride, Operand hidden, int vocab, int dim, const int32_t *count, int splits,
                                                          float *logits, int64_t logits_stride, int64_t split_stride) {
    constexpr int kMi = 4, kNj = kN / 16, kPlanes = Planes<F>::kCount, kSums = kPlanes > 1 ? 2 : 1;
    typedef typename T::Frag Frag;
    const int lane = threadIdx.x & 63, r = lane & 15, group = lane >> 4, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int first = (blockIdx.x * 4 + wave) * kMi * 16, rows = *count, split = blockIdx.y;
    if (first >= vocab) return;
    const int chunks = (dim + 31) / 32, begin = chunks * split / splits, end = chunks * (split + 1) / splits;
    const typename F::Stored *row[kMi];
    const char *of[kNj];
#pragma unroll
    for (int i = 0; i < kMi; ++i) row[i] = weight + min(first + i * 16 + r, vocab - 1) * weight_stride;
#pragma unroll
    for (int j = 0; j < kNj; ++j) of[j] = hidden.at + min(j * 16 + r, hidden.rows - 1) * hidden.stride + group * 16;
    Float4 acc[kSums][kMi][kNj];
#pragma unroll
    for (int s = 0; s < kSums; ++s)
#pragma unroll
        for (int i = 0; i < kMi; ++i)
#pragma unroll
            for (int j = 0; j < kNj; ++j) acc[s][i][j] = Float4{0, 0, 0, 0};
    Eight<F> a[2][kMi];
    auto load = [&](int which, int chunk) {
        const int k = chunk * 32 + group * 8;
#pragma unroll
        for (int i = 0; i < kMi; ++i) {
            if (k + 8 <= dim) a[which][i] = load_eight<F, false>(row[i], k / 8);
            else {
                float x[8];
                eight_of<F>(row[i], k, dim, x);
                a[which][i] = eight_from<F>(x);
            }
        }
    };
    auto multiply = [&](int which, int chunk) {
        Frag b[kPlanes][kNj];
#pragma unroll
        for (int p = 0; p < kPlanes; ++p)
#pragma unroll
            for (int j = 0; j < kNj; ++j) b[p][j] = *reinterpret_cast<const Frag *>(of[j] + p * hidden.plane + chunk * 64);
#pragma unroll
        for (int i = 0; i < kMi; ++i) {
            if constexpr (kPlanes == 1) {
                const Frag x = __builtin_bit_cast(Frag, a[which][i].v[0]);
#pragma unroll
                for (int j = 0; j < kNj; ++j) acc[0][i][j] = T::multiply(x, b[0][j], acc[0][i][j]);
            } else {
                const uint32_t w[8] = {a[which][i].v[0].x, a[which][i].v[0].y, a[which][i].v[0].z, a[which][i].v[0].w, a[which][i].v[1].x, a[which][i].v[1].y, a[which][i].v[1].z, a[which][i].v[1].w};
                float left[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) left[e] = __builtin_bit_cast(float, w[e]);
                Frag x[3];
#pragma unroll
                for (int p = 0; p < 3; ++p) x[p] = __builtin_bit_cast(Frag, take_plane<F>(left));
#pragma unroll
                for (int j = 0; j < kNj; ++j) {
                    acc[0][i][j] = T::multiply(x[0], b[0][j], acc[0][i][j]);
#pragma unroll
                    for (int pair = 0; pair < 5; ++pair) acc[1][i][j] = T::multiply(x[plane_of_a(6, pair)], b[plane_of_b(6, pair)][j], acc[1][i][j]);
                }
            }
        }
    };
    if (begin < end) load(0, begin);
#pragma nounroll
    for (int chunk = begin; chunk < end; chunk += 2) {
        if (chunk + 1 < end) load(1, chunk + 1);
        multiply(0, chunk);
        if (chunk + 1 >= end) break;
        if (chunk + 2 < end) load(0, chunk + 2);
        multiply(1, chunk + 1);
    }
#pragma unroll
    for (int j = 0; j < kNj; ++j) {
        const int n = j * 16 + r;
        if (n >= rows) continue;
        float *out = logits + split * split_stride + n * logits_stride;
#pragma unroll
        for (int i = 0; i < kMi; ++i) {
            const int v = first + i * 16 + group * 4;                     // (a row of logits has whole pieces of 16)
            Float4 sum = acc[0][i][j];
            if constexpr (kSums > 1) sum += acc[1][i][j];
            if (v < logits_stride) *reinterpret_cast<Float4 *>(out + v) = sum;
        }
    }
}

// ---- at most eight rows (vector_rows): vector instructions on 32-bit numbers, which read the weights as they lie, once for the logits and once for both gradients.

// The logits of kTokens tokens a wave.  A lane sums its eighth of every 512 numbers; at the end the lanes' sums are added in pairs, half of the results
// each time, until every lane has one.
constexpr int kFewTokens = 8;
template <int kLeft, int kApart>
__device__ __forceinline__ void fold(float *sum, int lane) {
    if constexpr (kApart > 0) {
        if constexpr (kLeft > 1) {
            const bool upper = lane & kApart;
#pragma unroll
            for (int i = 0; i < kLeft / 2; ++i) {
                const float keep = upper ? sum[i + kLeft / 2] : sum[i], give = upper ? sum[i] : sum[i + kLeft / 2];
                sum[i] = keep + __shfl_xor(give, kApart);
            }
            fold<kLeft / 2, kApart / 2>(sum, lane);
        } else {
            sum[0] += __shfl_xor(sum[0], kApart);
            fold<1, kApart / 2>(sum, lane);
        }
    }
}
template <class F, int kRows>
__global__ __launch_bounds__(256) void head_few_logits_kernel(const typename F::Stored *weight, int64_t weight_stride, const typename F::Stored *hidden, int64_t hidden_stride, const int32_t *count,
                                                              const int32_t *row_of, int vocab, int dim, float *logits, int64_t logits_stride) {
    const int lane = threadIdx.x & 63, first = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)) * kFewTokens), rows = *count;
    if (first >= vocab) return;
    constexpr int kResults = kFewTokens * kRows;
    float sum[kResults];
#pragma unroll
    for (int i = 0; i < kResults; ++i) sum[i] = 0.0f;
    // (waves begin at places of their own: rows a power of two apart lie in the same channels)
    const int columns = (dim + 511) / 512;
    for (int i = 0, column = first / kFewTokens % columns; i < columns; ++i, column = column + 1 == columns ? 0 : column + 1) {
        const int d = column * 512 + lane * 8;
        if (d >= dim) continue;
        float w[kFewTokens][8];
#pragma unroll
        for (int t = 0; t < kFewTokens; ++t) eight_of<F>(weight + min(first + t, vocab - 1) * weight_stride, d, dim, w[t]);
#pragma unroll
        for (int n = 0; n < kRows; ++n) {
            if (n >= rows) break;
            float h[8];
            eight_of<F>(hidden + row_of[n] * hidden_stride, d, dim, h);
#pragma unroll
            for (int t = 0; t < kFewTokens; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[t * kRows + n] = fmaf(w[t][e], h[e], sum[t * kRows + n]);
        }
    }
    fold<kResults, 32>(sum, lane);
    const int result = lane / (64 / kResults), n = result % kRows, v = first + result / kRows;
    if (lane % (64 / kResults) == 0 && n < rows && v < vocab) logits[n * logits_stride + v] = sum[0];
}

// Both gradients (null: not wanted): a block's eight waves take 512 numbers of the weights of every eighth 16 of its tokens, with the rows' slopes, which they
// make of the logits, and the hidden states in registers.  d weight is written at once; the sums of d hidden are added up over the waves, and the
// blocks' by the kernel behind.  Numbers that are not finite count as 0: a masked token's slope, zero, makes them nothing.
constexpr int kFewWaves = 8, kFewGroup = 16;
template <class F, int kRows>
__global__ __launch_bounds__(kFewWaves * 64) void head_few_grad_kernel(const typename F::Stored *weight, int64_t weight_stride, const typename F::Stored *hidden, int64_t hidden_stride,
                                                                       const float *logits, int64_t logits_stride, HeadMask mask, Taught taught, const float2 *stats, int dim, int tokens_of_block,
                                                                       float *sums, int64_t sums_stride, int64_t split_stride, typename F::Stored *out, int64_t out_stride) {
    __shared__ float waves[kFewWaves][512];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), d = blockIdx.y * 512 + lane * 8, rows = *taught.count;
    const int begin = blockIdx.x * tokens_of_block, end = min(mask.vocab, begin + tokens_of_block);
    auto finite = [](float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fabsf(x[e]) < INFINITY ? x[e] : 0.0f;
    };
    float h[kRows][8], sum[kRows][8], g[kRows], top[kRows], share[kRows];
    int target[kRows], row[kRows];
#pragma unroll
    for (int n = 0; n < kRows; ++n) {
        row[n] = n < rows ? taught.row[n] : 0;
        target[n] = n < rows ? taught.target[n] : -1;
        g[n] = n < rows ? taught.weight[n] : 0.0f;
        const float2 s = n < rows ? stats[row[n]] : make_float2(0.0f, 1.0f);
        top[n] = s.x;
        share[n] = 1.0f / s.y;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[n][e] = sum[n][e] = 0.0f;
        if (n < rows && out) eight_of<F>(hidden + row[n] * hidden_stride, d, dim, h[n]);
        finite(h[n]);
    }
    for (int v0 = begin + wave * kFewGroup; v0 < end; v0 += kFewWaves * kFewGroup) {
        // lane i: the slopes of the i-th token
        float slope[kRows];
        const int mine = v0 + lane % kFewGroup;
#pragma unroll
        for (int n = 0; n < kRows; ++n) {
            slope[n] = 0.0f;
            if (n >= rows || mine >= end) continue;
            if (mask.bitmask && !(mask.bitmask[(size_t)row[n] * mask.words + (mine >> 5)] >> (mine & 31) & 1u)) continue;
            slope[n] = (__builtin_amdgcn_exp2f((logits[n * logits_stride + mine] - top[n]) * kLog2E) * share[n] - (mine == target[n] ? 1.0f : 0.0f)) * g[n];
        }
        constexpr int kAtOnce = kRows < 8 ? 8 : 4;
#pragma unroll
        for (int t0 = 0; t0 < kFewGroup; t0 += kAtOnce) {
            float w[kAtOnce][8];
            if (sums)
#pragma unroll
                for (int t = 0; t < kAtOnce; ++t) {
                    eight_of<F>(weight + min(v0 + t0 + t, mask.vocab - 1) * weight_stride, min(d, (dim + 7) / 8 * 8), dim, w[t]);
                    finite(w[t]);
                }
#pragma unroll
            for (int t = 0; t < kAtOnce; ++t) {
                float y[8] = {};
#pragma unroll
                for (int n = 0; n < kRows; ++n) {
                    const float s = from_lane(slope[n], t0 + t);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (sums) sum[n][e] = fmaf(s, w[t][e], sum[n][e]);
                        if (out) y[e] = fmaf(s, h[n][e], y[e]);
                    }
                }
                if (out && v0 + t0 + t < end && d < dim) put_eight<F, true>(y, out + (v0 + t0 + t) * out_stride, d, dim);
            }
        }
    }
    if (!sums) return;
    for (int n = 0; n < kRows; ++n) {
        if (n >= rows) break;
        __syncthreads();
#pragma unroll
        for (int m = 0; m < kRows; ++m)                                   // (registers have no index)
            if (m == n)
#pragma unroll
                for (int e = 0; e < 8; ++e) waves[wave][lane * 8 + e] = sum[m][e];
        __syncthreads();
        float all = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) all += waves[w][threadIdx.x];
        const int column = blockIdx.y * 512 + threadIdx.x;
        if (column < sums_stride) sums[blockIdx.x * split_stride + n * sums_stride + column] = all;
    }
}

// A row of d hidden, or of d weight (place null: all rows are there), from the shares' and planes' sums, rounded once; zeros for rows that are not taught.  kGroups
// threads take every kGroups-th of them, and their sums are added in order.
template <class F, int kGroups>
__global__ __launch_bounds__(256) void head_sums_join_kernel(const int32_t *place, const int32_t *count, const float *scale, const float *sums, Shares shares, int planes, int64_t sums_stride,
                                                               int64_t split_stride, int64_t plane_stride, int dim, typename F::Stored *out, int64_t out_stride) {
    constexpr int kFours = 256 / kGroups;
    __shared__ Float4 parts[kGroups][kFours];
    const int r = blockIdx.x, at = place ? place[r] : r, four = threadIdx.x % kFours, group = threadIdx.x / kFours, d = (blockIdx.y * kFours + four) * 4;
    const int all = planes * (shares.tiles_m ? shares_of(shares.tiles_m, shares.tile_n, *count, shares.blocks, shares.most) : shares.most);
    Float4 x = {0, 0, 0, 0};
    if (at >= 0 && d < dim)
        for (int s = group; s < all; s += kGroups) x += *reinterpret_cast<const Float4 *>(sums + s / planes * split_stride + s % planes * plane_stride + at * sums_stride + d);
    if constexpr (kGroups > 1) {
        parts[group][four] = x;
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int g = 1; g < kGroups; ++g) x += parts[g][four];
    }
    if (d >= dim) return;
    x *= scale[1];
    typename F::Stored *to = out + r * out_stride + d;
    if (d + 4 <= dim) {
        if constexpr (sizeof(typename F::Stored) == 2) {
            typedef uint2 __attribute__((aligned(2))) Unaligned;
            *reinterpret_cast<Unaligned *>(to) = at < 0 ? make_uint2(0, 0) : make_uint2(F::pair(x[0], x[1]), F::pair(x[2], x[3]));
        } else {
            *reinterpret_cast<UnalignedUint4 *>(to) = at < 0 ? UnalignedUint4{0, 0, 0, 0} : UnalignedUint4{F::pattern(x[0]), F::pattern(x[1]), F::pattern(x[2]), F::pattern(x[3])};
        }
    } else {
        for (int e = 0; d + e < dim; ++e) to[e] = at < 0 ? (typename F::Stored)0 : (typename F::Stored)F::pattern(x[e]);
    }
}

// d weight of a piece of the vocabulary, whole: out[token][dim].
template <class T, class F, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head_weight_grad_kernel(Operand hidden, Operand slopes, int pairs, int tiles_m, int tiles_n, const int32_t *count, const int32_t *infinite,
                                                                          const float *scale, int dim, int tokens, typename F::Stored *out, int64_t out_stride) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int k_steps = (*count + kStepRows - 1) / kStepRows, steps = k_steps * pairs;
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
    run_finite(tile, infinite, hidden, slopes, pairs, max(k_steps, 1), lds, tiles, [&](const TileAt &at) {
#pragma unroll
        for (int j = 0; j < Tile::kNj; ++j) {
            const int v = at.n0 + Tile::n_of(j);
            if (v >= tokens) continue;
#pragma unroll
            for (int i = 0; i < Tile::kMi; i += 2) {
                float x[8];
                const int d = at.m0 + tile.eight_of_lane(i, j, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= back;
                put_eight<F, false>(x, out + v * out_stride, d, dim);
            }
        }
    });
}

template <class S>
__global__ __launch_bounds__(256) void zero_rows_kernel(S *at, int dim, int64_t stride) {
    for (int d = blockIdx.y * 256 + threadIdx.x; d < dim; d += gridDim.y * 256) at[blockIdx.x * stride + d] = 0;
}

// ------------------------------------------------------------------------------------------------- host

size_t up(size_t n, size_t to) { return (n + to - 1) / to * to; }

// Tiles by their rows.  us of one product, 4,096 numbers a row in bf16 (TB/s or TFLOP/s): 57,344 tokens and 32 rows in tiles of 128 x 32 86 (5.5),
// 256 x 32 98; 64 rows in 256 x 64 87 (5.4), 128 x 64 93, 64 x 64 103; 128 rows in 256 x 128 by eight waves 96 (4.9), by four 108, 128 x 128 106;
// 42,752 tokens and 3,840 rows in 256 x 256 1,190 (1,130), 256 x 128 1,330 (1,010), 128 x 128 1,760, 256 x 256 by four waves 1,860.
enum Form { kFew, kRows32, kRows64, kRows128, kRows256 };
template <class T, bool kColumnsA, bool kColumnsB, class Fn>
hipError_t with_tile(int form, Fn fn) {
    switch (form) {
        case kFew: return fn((ProductTile<T, 64, 64, 1, 2, 4, kColumnsA, kColumnsB> *)nullptr);
        case kRows32: return fn((ProductTile<T, 128, 32, 2, 1, 4, kColumnsA, kColumnsB> *)nullptr);
        case kRows64: return fn((ProductTile<T, 256, 64, 4, 1, 3, kColumnsA, kColumnsB> *)nullptr);
        case kRows128: return fn((ProductTile<T, 256, 128, 4, 2, 3, kColumnsA, kColumnsB> *)nullptr);
        default: return fn((ProductTile<T, 256, 256, 4, 2, 2, kColumnsA, kColumnsB> *)nullptr);
    }
}
// The forms that take rows as they come, with the logits in the tiles.
template <class T, class Fn>
hipError_t with_large_tile(int form, Fn fn) {
    return form == kRows128 ? fn((ProductTile<T, 256, 128, 4, 2, 3> *)nullptr) : fn((ProductTile<T, 256, 256, 4, 2, 2> *)nullptr);
}
// Which form a product m x n takes, and in how many shares along k: the cheapest by what a step of a tile takes, alone (us) or where all units fetch
// (8.3 TB/s; both measured), three us a launch, and the splits' sums, written and read at 3 TB/s.  (In columns a step of 64 x 64 takes 0.65 us; where few
// tiles leave units idle it is the cheapest form all the same: d weight of 2,000 rows, 600 tokens and 2,048 f32 numbers 126 us, 256 x 128 150.)
struct Choice { int form, splits; double us; };
Choice choose(size_t m, size_t n, int steps, bool split, int from, int to) {
    struct { int m, n, units; double alone; } const forms[] = {{64, 64, 2 * kUnits, 0.43}, {128, 32, 2 * kUnits, 0.46}, {256, 64, kUnits, 0.79}, {256, 128, kUnits, 0.78}, {256, 256, kUnits, 1.3}};
    Choice best{from, 1, 1e30};
    for (int f = from; f <= to; ++f) {
        const auto &form = forms[f];
        const size_t tiles = (m + form.m - 1) / form.m * ((n + form.n - 1) / form.n);
        for (int splits = 1; splits <= 256; splits += (splits + 3) / 4) {
            if (splits > 1 && (!split || steps / splits < 4)) break;
            const size_t blocks = tiles * splits, turns = (blocks + form.units - 1) / form.units;
            const double at_once = (double)std::min<size_t>(blocks, form.units), step = std::max(form.alone, at_once * (form.m + form.n) * kStepBytes / 8.3e6);
            const double us = 3 + (double)turns * ((steps + splits - 1) / splits * step + 1) + (split ? (double)splits * m * n * 8 / 3e6 : 0);
            if (us < best.us) best = {f, splits, us};
        }
    }
    return best;
}
int rows_of_form(int form) { return form == kRows32 ? 32 : form == kFew || form == kRows64 ? 64 : form == kRows128 ? 128 : 256; }

// Where everything lies in the workspace, and how the vocabulary is cut.
struct Plan {
    int planes, slope_planes, padded_rows, pieces, piece; // tokens of a piece: a multiple of kMostTokens
    bool packs_weight;                                   // the weights' rows are not as the products read them
    bool few, few_logits, by_rows, direct;               // at most vector_rows, the logits as well; the logits are kept for the call; from weights as they lie
    int dim_bytes, piece_bytes;                          // of a plane of a packed row of hidden states and weights, and of one of slopes
    Choice logits, hidden, tokens;                       // of the logits, of d hidden, and of d weight
    int few_tokens;                                      // of a block, of few rows
    int part_tokens, n_parts, parts_stride;              // of which maximum and sum come out together
    int plane_rows;                                      // the second plane of slopes are further rows, from this one on (0: planes lie in the rows)
    int64_t logits_stride, logits_split, sums_stride, sums_split, weight_split;
    size_t count, infinite, scale, place, row, target, weight, target_logit, parts, packed_hidden, packed_weight, stats, logits_at, slopes, sums, weight_sums, bytes;
};
constexpr int kMostTokens = 256;                         // of a tile
constexpr size_t kPieceBytes = (size_t)1 << 30;
// Slopes are summed over all rows, or all tokens.  Roundings of many rows' slopes come out as one of them does, beside that of the result; of few
// rows a gradient can have one slope's, whole.  These have slopes of two parts, 16 or 22 bits: their products wait for memory in any case.
constexpr int kFewRows = 128;
// Rows that vector instructions multiply while the weights are on their way.  us of loss and gradients, so and by matrix instructions (which read weights that
// lie otherwise three times more): 52,374 x 1,216 bf16, 2 rows 133 and 133, 4 rows 160 and 133, 8 rows 447 and 134; 100,003 x 1,001 f16, 4 rows 265 and 296,
// 5 rows 789 and 295 (there are no registers for more); 50,000 x 1,024 f32, 4 rows 169 and 429.  The rule knows types and rows only, not what is wanted: 8 rows of the f32 head
// take 490 and 430 with gradients, their loss alone 49 and 78.
constexpr int vector_rows(int planes, bool packs_weight) { return planes > 1 ? 8 : packs_weight ? 4 : 2; }

// Rows and numbers of weights of which a loss alone is taken from weights as they lie.  us, packed first and as they lie: 16 rows of 128,256 x 2,048 f32
// 1,036 and 331, 40 of 8,000 x 1,001 51 and 41, 64 of 2,000 x 1,001 32 and 31; packed 16-bit weights stay in the caches up to some size: 40 rows of
// 100,003 x 1,001 f16 150 and 105, 64 of 50,257 x 769 bf16 61 and 76.
constexpr int kDirectRows = 64;
constexpr int64_t direct_numbers(int planes) { return planes > 1 ? 1 << 20 : 1 << 26; }

// alone: of a loss that leaves nothing to a backward pass.
Plan plan_of(const HeadRows &h, bool grads, bool alone) {
    Plan p{};
    p.planes = h.type == kLogitF32 ? 3 : 1;
    p.slope_planes = p.planes > 1 ? 3 : h.rows <= kFewRows ? 2 : 1;
    const size_t size = h.type == kLogitF32 ? 4 : 2;
    p.packs_weight = p.planes > 1 || h.dim % 8 != 0 || (reinterpret_cast<uintptr_t>(h.weight) | (uintptr_t)(h.weight_stride * size)) % 16 != 0 || h.weight_stride >= 1 << 22;
    p.dim_bytes = (int)up((size_t)h.dim * 2, kStepBytes);
    const int pairs = pairs_of(p.planes, p.planes), dim_steps = p.dim_bytes / kStepBytes * pairs;
    // Rows by rows where they are few, and where a split product with its logits' way to memory and back is cheaper than tiles of rows as they come.  (Of the forward pass: what
    // kept logits spare a backward pass is not in the comparison.)
    const Choice tiles = choose(h.vocab, h.rows, dim_steps, false, kRows128, kRows256), split = choose(h.vocab, h.rows, dim_steps, true, kFew, kRows256);
    const double logits_us = 4 + (double)h.rows * h.vocab * 8 / 3e6;
    p.few = h.rows <= vector_rows(p.planes, p.packs_weight);
    p.by_rows = h.rows <= kFewRows || ((double)split.splits * h.rows * h.vocab * 4 < kPieceBytes / 4 && split.us + logits_us < tiles.us);
    p.logits = p.by_rows ? split : tiles;
    p.padded_rows = (int)up(h.rows, std::max(rows_of_form(p.logits.form), kStepRows));
    // (weights that lie as the products read them are streamed faster by these: 128,256 x 4,096 bf16 and one row 176 us, with vector instructions 197)
    p.few_logits = p.few && p.packs_weight;
    if (p.few_logits) p.logits.splits = 1;
    p.direct = alone && p.packs_weight && !p.few && h.rows <= kDirectRows && (int64_t)h.vocab * h.dim >= direct_numbers(p.planes);
    if (p.direct) p.logits.splits = std::max(1, std::min(2 * kUnits / ((h.vocab + 255) / 256), (h.dim + 31) / 32 / 4));      // eight waves a unit, of four chunks and more
    // what a token takes while its piece is worked on
    const size_t each = p.few || p.direct ? 0 : (p.packs_weight ? (size_t)p.planes * p.dim_bytes : 0) + (grads ? 2 * (size_t)p.slope_planes * p.padded_rows : 0);
    const size_t most = each ? std::max<size_t>(kMostTokens, kPieceBytes / each / kMostTokens * kMostTokens) : up(h.vocab, kMostTokens);
    p.pieces = (int)((h.vocab + most - 1) / most);
    p.piece = (int)up((h.vocab + p.pieces - 1) / p.pieces, kMostTokens);
    p.pieces = (h.vocab + p.piece - 1) / p.piece;
    p.piece_bytes = p.piece * 2;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t from = at; at += up(bytes, 256); return from; };
    p.count = take(4);
    p.infinite = take(4);
    p.scale = take(8);
    for (size_t *x : {&p.place, &p.row, &p.target, &p.weight, &p.target_logit}) *x = take((size_t)h.rows * 4);
    p.stats = take((size_t)h.rows * 8);
    if (!p.few_logits) p.packed_hidden = take((size_t)p.padded_rows * p.planes * p.dim_bytes);
    if (p.packs_weight && !p.few && !p.direct) p.packed_weight = take((size_t)p.piece * p.planes * p.dim_bytes);
    if (p.by_rows) {                                     // of the whole vocabulary: both passes of a call have them
        p.logits_stride = (int64_t)up(h.vocab, kLaneTokens);
        p.logits_split = p.logits_stride * h.rows;
        p.logits_at = take((size_t)p.logits.splits * p.logits_split * 4);
    }
    // parts of a row: its waves' shares of tiles, or stretches of its logits, as long as there are two blocks for every unit
    p.part_tokens = p.by_rows ? (int)up(std::max<int64_t>(1, (int64_t)h.vocab * h.rows / (2 * kUnits)), kRowTokens) : kPartTokens;
    p.n_parts = (h.vocab + p.part_tokens - 1) / p.part_tokens;
    p.parts_stride = p.padded_rows;
    const size_t parts_bytes = (p.by_rows ? p.n_parts : up(h.vocab, kMostTokens) / kPartTokens) * (size_t)p.parts_stride * 8;
    if (p.by_rows) p.parts = take(parts_bytes);
    const size_t both = at;
    if (!p.by_rows) p.parts = take(parts_bytes);
    p.sums_stride = (int64_t)up(h.dim, kLaneTokens);
    if (grads && p.few) {
        // a block takes 512 numbers of each of so many tokens: four blocks and more for every unit
        const int64_t columns = (h.dim + 511) / 512;
        p.few_tokens = (int)up(std::max<int64_t>(1, h.vocab * columns / (4 * kUnits)), kFewWaves * kFewGroup);
        p.hidden = {0, (h.vocab + p.few_tokens - 1) / p.few_tokens, 0};
        p.sums_split = p.sums_stride * h.rows;
        p.sums = take((size_t)p.hidden.splits * p.sums_split * 4);
    } else if (grads) {
        const size_t forward = at;
        at = both;                                       // (the parts have been joined by then)
        p.plane_rows = p.slope_planes == 2 ? (int)up(h.rows, kStepRows) : 0;
        const int n = p.plane_rows ? 2 * p.plane_rows : h.rows, steps = p.piece_bytes / kStepBytes * (p.planes > 1 ? pairs : 1);
        p.hidden = choose(h.dim, n, steps, true, kFew, kRows256);
        p.sums_split = p.sums_stride * n;
        // (not all rows are taught: with half of them there are twice the shares)
        if (!p.plane_rows) p.hidden.splits = std::max(1, (int)std::min<int64_t>({2 * p.hidden.splits, steps / 4, std::max<int64_t>(p.hidden.splits, (int64_t)(kPieceBytes / 4) / (p.sums_split * 4))}));
        // (a step of rows is read along them as well)
        p.slopes = take((p.plane_rows ? 2 * (size_t)p.plane_rows : (size_t)p.padded_rows * p.slope_planes) * p.piece_bytes);
        p.sums = take((size_t)p.hidden.splits * p.sums_split * 4);
        // d weight, of few tokens in shares along the rows (4,346 rows of 143 tokens and 154 bf16 numbers: 40 -> 12 us with their sums' way to memory and back)
        const int weight_steps = p.padded_rows / kStepRows * pairs_of(p.planes, p.slope_planes);
        p.tokens = choose(h.dim, p.piece, weight_steps, false, kFew, kRows256);
        const Choice shares = choose(h.dim, p.piece, weight_steps, true, kFew, kRows256);
        p.weight_split = p.sums_stride * p.piece;
        if (shares.splits > 1 && shares.us + 4 < p.tokens.us && (size_t)shares.splits * p.weight_split * 4 <= kPieceBytes / 4) {
            p.tokens = shares;
            p.weight_sums = take((size_t)shares.splits * p.weight_split * 4);
        }
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
    return {w.as<int32_t>(p.count), w.as<int32_t>(p.infinite), w.as<float>(p.scale), w.as<int32_t>(p.place), w.as<int32_t>(p.row), w.as<int32_t>(p.target), w.as<float>(p.weight)};
}

// A block takes a unit to itself, or shares it with others where they fit.
template <class Tile>
int blocks_of(int tiles) { return std::min(tiles, kUnits * (160 * 1024 / Tile::kLdsBytes)); }
template <class Tile, class Kernel, class... Args>
hipError_t launch_tiles(Kernel kernel, int tiles, hipStream_t stream, Args... args) {
    constexpr int threads = Tile::kThreads, lds = Tile::kLdsBytes;
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(blocks_of<Tile>(tiles)), dim3(threads), lds, stream, args...);
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

    Head(const HeadRows &h_, bool grads, bool alone, void *workspace, hipStream_t stream_)
        : h(h_), p(plan_of(h_, grads, alone)), w{static_cast<char *>(workspace)}, taught(taught_of(p, w)), mask{h_.bitmask, h_.vocab, (h_.vocab + 31) / 32}, stream(stream_) {}

    const Stored *weight_at(int v0) const { return static_cast<const Stored *>(h.weight) + (int64_t)v0 * h.weight_stride; }
    int tokens_of(int v0) const { return std::min(p.piece, h.vocab - v0); }
    Pack pack_hidden(bool wanted) const {
        return {h.hidden, h.hidden_stride, taught.row, taught.count, h.rows, h.dim, p.padded_rows, wanted ? w.as<char>(p.packed_hidden) : nullptr, p.dim_bytes};
    }
    Pack pack_weight(int v0) const {
        const int tokens = tokens_of(v0);
        return {weight_at(v0), h.weight_stride, nullptr, nullptr, tokens, h.dim, tokens, p.packs_weight ? w.as<char>(p.packed_weight) : nullptr, p.dim_bytes};
    }
    Operand hidden() const { return {w.as<char>(p.packed_hidden), (int64_t)p.planes * p.dim_bytes, p.padded_rows, p.dim_bytes, p.dim_bytes}; }
    Operand weight(int v0) const {
        if (!p.packs_weight) return {reinterpret_cast<const char *>(weight_at(v0)), h.weight_stride * 2, tokens_of(v0), h.dim * 2, 0};
        return {w.as<char>(p.packed_weight), (int64_t)p.planes * p.dim_bytes, tokens_of(v0), p.dim_bytes, p.dim_bytes};
    }
    Slopes slopes_to() const {
        if (p.plane_rows) return {w.as<char>(p.slopes), p.piece_bytes, (int64_t)p.plane_rows * p.piece_bytes};
        return {w.as<char>(p.slopes), (int64_t)p.slope_planes * p.piece_bytes, p.piece_bytes};
    }
    // The slopes of a piece, along the tokens or (in columns) the rows.
    Operand slopes_of(int rows) const {
        const Slopes to = slopes_to();
        return {to.at, to.row_stride, rows, p.piece_bytes, (int)to.plane};
    }
    int pairs() const { return pairs_of(p.planes, p.planes); }
    // The logits of rows by rows, where the products write them, in splits, and where they are added up: kept from the loss's call to the gradients' if asked for.
    float *all_logits() const { return h.kept ? h.kept : w.as<float>(p.logits_at); }
    float *sums_of_logits() const { return p.logits.splits > 1 ? w.as<float>(p.logits_at) : all_logits(); }

    // Logits of a piece, or what remains of them.
    hipError_t logits(int v0) const {
        const int tokens = tokens_of(v0), k_steps = p.dim_bytes / kStepBytes;
        if (p.by_rows)
            return with_tile<T, false, false>(p.logits.form, [&](auto *tile) {
                typedef std::remove_pointer_t<decltype(tile)> Tile;
                return launch_sums<Tile>(weight(v0), hidden(), pairs(), k_steps, p.logits.splits, tokens, h.rows, taught.count, nullptr, sums_of_logits() + v0, p.logits_stride, p.logits_split,
                                         (int)up(tokens, kLaneTokens), true, false);
            });
        return with_large_tile<T>(p.logits.form, [&](auto *tile) {
            typedef std::remove_pointer_t<decltype(tile)> Tile;
            const int tiles_m = (tokens + Tile::kM - 1) / Tile::kM;
            return launch_tiles<Tile>(head_stats_kernel<T, Tile>, tiles_m * (p.padded_rows / Tile::kN), stream, weight(v0), hidden(), pairs(), k_steps, v0, tiles_m, mask,
                                      (const int32_t *)taught.count, (const int32_t *)taught.row, (const int32_t *)taught.target, w.as<float2>(p.parts), p.parts_stride,
                                      w.as<float>(p.target_logit));
        });
    }
    template <int kN>
    hipError_t direct_logits() const {
        hipLaunchKernelGGL((head_direct_kernel<T, F, kN>), dim3((h.vocab + 255) / 256, p.logits.splits), dim3(256), 0, stream, weight_at(0), h.weight_stride, hidden(), h.vocab,
                           h.dim, taught.count, p.logits.splits, sums_of_logits(), p.logits_stride, p.logits_split);
        return hipGetLastError();
    }
    hipError_t direct_logits() const {
        return h.rows <= 32 ? direct_logits<32>() : direct_logits<64>();
    }
    hipError_t rows(float *loss, float *stats) const {
        const bool whole = p.by_rows && p.n_parts == 1;
        if (p.by_rows)
            hipLaunchKernelGGL(head_row_kernel, dim3(h.rows, p.n_parts), dim3(kRowThreads), 0, stream, taught.place, mask, taught.target, sums_of_logits(), p.logits_stride,
                               p.logits_split, p.logits.splits, all_logits(), p.part_tokens, whole ? nullptr : w.as<float2>(p.parts), p.parts_stride, w.as<float>(p.target_logit), loss, reinterpret_cast<float2 *>(stats));
        if ((loss || stats) && !whole)
            hipLaunchKernelGGL(head_join_kernel, dim3((h.rows + kJoinRows - 1) / kJoinRows), dim3(1024), 0, stream, taught.place, h.rows, w.as<float2>(p.parts), p.parts_stride,
                               p.n_parts, w.as<float>(p.target_logit), loss, reinterpret_cast<float2 *>(stats));
        return hipGetLastError();
    }
    template <int kPlanes>
    hipError_t slopes(int v0, const float *stats, const Slopes &out) const {
        const int tokens = tokens_of(v0);
        if (p.by_rows) {
            hipLaunchKernelGGL((head_row_slopes_kernel<Part, kPlanes>), dim3((tokens + 63) / 64, p.padded_rows / 64), dim3(256), 0, stream, all_logits(), p.logits_stride, v0, mask,
                               taught, reinterpret_cast<const float2 *>(stats), p.plane_rows ? p.plane_rows : p.padded_rows, out);
            return hipGetLastError();
        }
        if constexpr (kPlanes == 2) return hipErrorInvalidValue;        // (few rows have their logits)
        else
            return with_large_tile<T>(p.logits.form, [&](auto *tile) {
                typedef std::remove_pointer_t<decltype(tile)> Tile;
                const int tiles_m = (tokens + Tile::kM - 1) / Tile::kM;
                return launch_tiles<Tile>(head_slopes_kernel<T, Part, Tile, kPlanes>, tiles_m * (p.padded_rows / Tile::kN), stream, weight(v0), hidden(), pairs(), p.dim_bytes / kStepBytes, v0,
                                          tiles_m, mask, taught, reinterpret_cast<const float2 *>(stats), out);
            });
    }
    hipError_t slopes(int v0, const float *stats, const Slopes &out) const {
        if constexpr (sizeof(Stored) == 4) return slopes<3>(v0, stats, out);
        else return p.slope_planes == 2 ? slopes<2>(v0, stats, out) : slopes<1>(v0, stats, out);
    }
    template <class Tile>
    hipError_t launch_sums(const Operand &a, const Operand &b, int pairs, int k_steps, int splits, int m, int n, const int32_t *rows, const int32_t *along, float *sums, int64_t stride, int64_t split_stride, int sums_m,
                           bool first, bool fitted) const {
        const int tiles_m = (m + Tile::kM - 1) / Tile::kM;
        return launch_tiles<Tile>(head_sums_kernel<T, Tile>, tiles_m * splits * ((n + Tile::kN - 1) / Tile::kN), stream, a, b, pairs, k_steps, splits, tiles_m, rows,
                                  along, (const int32_t *)taught.infinite, sums, stride, split_stride, sums_m, n, first, fitted);
    }
    // (the weights in columns: as they lie)
    hipError_t hidden_grad(int v0) const {
        const bool stacked = p.plane_rows > 0;
        const int rows = stacked ? 2 * p.plane_rows : p.padded_rows;
        return with_tile<T, true, false>(p.hidden.form, [&](auto *tile) {
            typedef std::remove_pointer_t<decltype(tile)> Tile;
            return launch_sums<Tile>(weight(v0), slopes_of(rows), stacked ? 1 : pairs_of(p.planes, p.slope_planes), (tokens_of(v0) + kStepRows - 1) / kStepRows, p.hidden.splits, h.dim,
                                     stacked ? rows : h.rows, stacked ? nullptr : taught.count, nullptr, w.as<float>(p.sums), p.sums_stride, p.sums_split, (int)p.sums_stride, v0 == 0, !stacked);
        });
    }
    // (hidden states and slopes in columns)
    hipError_t weight_grad(int v0, Stored *out, int64_t out_stride) const {
        const int tokens = tokens_of(v0), pairs = pairs_of(p.planes, p.slope_planes);
        return with_tile<T, true, true>(p.tokens.form, [&](auto *tile) {
            typedef std::remove_pointer_t<decltype(tile)> Tile;
            if (p.tokens.splits > 1) {
                const hipError_t e = launch_sums<Tile>(hidden(), slopes_of(p.plane_rows ? p.plane_rows : p.padded_rows), pairs, 0, p.tokens.splits, h.dim, tokens, nullptr, taught.count,
                                                       w.as<float>(p.weight_sums), p.sums_stride, p.weight_split, (int)p.sums_stride, true, false);
                if (e != hipSuccess) return e;
                return join(nullptr, tokens, w.as<float>(p.weight_sums), p.weight_split, Shares{0, 0, 0, p.tokens.splits}, 1, out + (int64_t)v0 * out_stride, out_stride);
            }
            const int tiles_d = (h.dim + Tile::kM - 1) / Tile::kM, tiles_v = (tokens + Tile::kN - 1) / Tile::kN;
            return launch_tiles<Tile>(head_weight_grad_kernel<T, F, Tile>, tiles_d * tiles_v, stream, hidden(), slopes_of(p.plane_rows ? p.plane_rows : p.padded_rows), pairs, tiles_d, tiles_v,
                                      (const int32_t *)taught.count, (const int32_t *)taught.infinite, (const float *)taught.scale, h.dim, tokens, out + (int64_t)v0 * out_stride, out_stride);
        });
    }

    template <class Fn>
    static hipError_t with_rows(int rows, Fn fn) {
        if (rows <= 1) return fn(std::integral_constant<int, 1>());
        if (rows <= 2) return fn(std::integral_constant<int, 2>());
        if constexpr (vector_rows(Planes<F>::kCount, true) == 8)
            if (rows > 4) return fn(std::integral_constant<int, 8>());
        return fn(std::integral_constant<int, 4>());
    }
    hipError_t few_logits() const {
        return with_rows(h.rows, [&](auto rows) {
            hipLaunchKernelGGL((head_few_logits_kernel<F, decltype(rows)::value>), dim3((h.vocab + 4 * kFewTokens - 1) / (4 * kFewTokens)), dim3(256), 0, stream, weight_at(0), h.weight_stride,
                               static_cast<const Stored *>(h.hidden), h.hidden_stride, taught.count, taught.row, h.vocab, h.dim, sums_of_logits(), p.logits_stride);
            return hipGetLastError();
        });
    }
    hipError_t few_grads(const float *stats, bool hidden, Stored *out, int64_t out_stride) const {
        return with_rows(h.rows, [&](auto rows) {
            hipLaunchKernelGGL((head_few_grad_kernel<F, decltype(rows)::value>), dim3(p.hidden.splits, (h.dim + 511) / 512), dim3(kFewWaves * 64), 0, stream, weight_at(0), h.weight_stride,
                               static_cast<const Stored *>(h.hidden), h.hidden_stride, all_logits(), p.logits_stride, mask, taught, reinterpret_cast<const float2 *>(stats), h.dim,
                               p.few_tokens, hidden ? w.as<float>(p.sums) : nullptr, p.sums_stride, p.sums_split, out, out_stride);
            return hipGetLastError();
        });
    }
    hipError_t join(const int32_t *place, int rows, const float *sums, int64_t split, const Shares &shares, int planes, Stored *out, int64_t out_stride) const {
        auto launch = [&](auto groups) {
            constexpr int kGroups = decltype(groups)::value;
            hipLaunchKernelGGL((head_sums_join_kernel<F, kGroups>), dim3(rows, (h.dim * kGroups + 1023) / 1024), dim3(256), 0, stream, place, taught.count, taught.scale, sums, shares, planes,
                               p.sums_stride, split, p.plane_rows * p.sums_stride, h.dim, out, out_stride);
            return hipGetLastError();
        };
        return shares.most > 8 ? launch(std::integral_constant<int, 16>()) : launch(std::integral_constant<int, 1>());
    }
    hipError_t hidden_join(Stored *out, int64_t out_stride) const {
        Shares shares{0, 0, 0, p.hidden.splits};
        if (!p.few && !p.plane_rows)
            (void)with_tile<T, true, false>(p.hidden.form, [&](auto *tile) {
                typedef std::remove_pointer_t<decltype(tile)> Tile;
                const int tiles_m = (h.dim + Tile::kM - 1) / Tile::kM;
                shares = {tiles_m, Tile::kN, blocks_of<Tile>(tiles_m * p.hidden.splits * ((h.rows + Tile::kN - 1) / Tile::kN)), p.hidden.splits};
                return hipSuccess;
            });
        return join(taught.place, h.rows, w.as<float>(p.sums), p.sums_split, shares, p.plane_rows ? 2 : 1, out, out_stride);
    }

    hipError_t run(bool forward, bool backward, float *loss, float *stats, const float *row_weight, int64_t weight_stride, Stored *grad_hidden, int64_t grad_hidden_stride,
                   Stored *grad_weight, int64_t grad_weight_stride) const {
        hipError_t e = hipSuccess;
        auto step = [&](hipError_t of) { return (e = of) == hipSuccess; };
        const bool whole = p.pieces == 1, kept = p.by_rows && h.kept && !forward;       // the loss's call has left the logits
        if (!stats) stats = w.as<float>(p.stats);
        hipLaunchKernelGGL(head_rows_kernel, dim3(1), dim3(kRowsThreads), 0, stream, h.targets, h.target_bytes, h.bitmask, h.rows, h.vocab, taught, backward, row_weight, weight_stride,
                           h.type == kLogitF16 && !p.few);
        if (p.few) {
            if (!kept && (p.few_logits ? !step(few_logits()) : !step(launch_pack<F>(pack_hidden(true), pack_weight(0), stream)) || !step(logits(0)))) return e;
            if ((forward || (p.logits.splits > 1 && !kept)) && !step(rows(forward ? loss : nullptr, forward ? stats : nullptr))) return e;
            if (!backward) return hipGetLastError();
            if (!step(few_grads(stats, grad_hidden != nullptr, grad_weight, grad_weight_stride))) return e;
            return grad_hidden ? hidden_join(grad_hidden, grad_hidden_stride) : hipSuccess;
        }
        // The logits, for the loss or for a backward pass of rows by rows (whose splits the loss's kernel adds up).
        const bool logits_first = forward || (p.by_rows && !kept);
        if (logits_first && p.direct) {
            if (!step(launch_pack<F>(pack_hidden(true), Pack{}, stream)) || !step(direct_logits())) return e;
        } else if (logits_first) {
            for (int v0 = 0; v0 < h.vocab; v0 += p.piece)           // (a vocabulary in one piece is packed once for both passes)
                if (!step(launch_pack<F>(pack_hidden(v0 == 0), pack_weight(v0), stream)) || !step(logits(v0))) return e;
        }
        if (logits_first && (forward || p.logits.splits > 1) && !step(rows(forward ? loss : nullptr, forward ? stats : nullptr))) return e;
        if (!backward) return hipGetLastError();
        for (int v0 = 0; v0 < h.vocab; v0 += p.piece) {
            const bool unread = p.by_rows && !grad_hidden;          // the weights
            if (!(logits_first && whole) && !step(launch_pack<F>(pack_hidden(!logits_first && v0 == 0), unread ? Pack{} : pack_weight(v0), stream))) return e;
            if (!step(slopes(v0, stats, slopes_to()))) return e;
            if (grad_hidden && !step(hidden_grad(v0))) return e;
            if (grad_weight && !step(weight_grad(v0, grad_weight, grad_weight_stride))) return e;
        }
        if (grad_hidden && !step(hidden_join(grad_hidden, grad_hidden_stride))) return e;
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

size_t head_call_bytes(const HeadRows &h, bool backward, bool alone) { return plan_of(h, backward, alone).bytes; }
size_t head_workspace_bytes(const HeadRows &h, HeadCalls calls) {
    // (the loss's calls may cut the vocabulary into fewer pieces: one workspace serves all calls)
    const size_t alone = plan_of(h, false, true).bytes;
    if (calls == HeadCalls::kLossAlone) return alone;
    const size_t loss = std::max(alone, plan_of(h, false, false).bytes);
    return calls == HeadCalls::kLoss ? loss : std::max(loss, plan_of(h, true, false).bytes);
}
size_t head_kept_bytes(const HeadRows &h) {
    const Plan p = plan_of(h, false, false);
    return p.by_rows ? (size_t)p.logits_split * 4 : 0;
}

hipError_t launch_head(const HeadRows &h, bool forward, bool backward, float *loss, float *stats, const float *row_weight, int64_t weight_stride, void *grad_hidden,
                       int64_t grad_hidden_stride, void *grad_weight, int64_t grad_weight_stride, void *workspace, hipStream_t stream) {
    auto run = [&](const auto &head) {
        typedef typename std::decay_t<decltype(head)>::Stored Stored;
        return head.run(forward, backward, loss, stats, row_weight, weight_stride, static_cast<Stored *>(grad_hidden), grad_hidden_stride, static_cast<Stored *>(grad_weight), grad_weight_stride);
    };
    const bool alone = !backward && head_is_alone(h, forward, stats);
    switch (h.type) {
        case kLogitBf16: return run(Head<ProductBf16, LogitsBf16>(h, backward, alone, workspace, stream));
        case kLogitF16: return run(Head<ProductF16, LogitsF16>(h, backward, alone, workspace, stream));
        default: return run(Head<ProductBf16, LogitsF32>(h, backward, alone, workspace, stream));
    }
}

}  // namespace pre3
