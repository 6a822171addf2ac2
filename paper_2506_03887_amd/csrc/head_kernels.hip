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

// What a tile's kernels know of the rows' side.
struct HeadMask {
    const uint32_t *bitmask;       // null: every token is allowed
    int vocab, words;
};
// The allowed tokens among the 128 from `v` on (a multiple of 32), of the taught row at place n.
template <int kWords>
__device__ __forceinline__ void allowed_words(const HeadMask &mask, const int32_t *row_of, int n, int v, uint32_t out[kWords]) {
    const uint32_t *words = mask.bitmask ? mask.bitmask + (size_t)row_of[n] * mask.words : nullptr;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        const int left = mask.vocab - (v + 32 * i);                       // tokens there are from this word on
        uint32_t w = left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
        if (words && left > 0) w &= words[(v >> 5) + i];
        out[i] = w;
    }
}

// Maximum, and sum of the exponentials over it, of every taught row over a wave's share of a tile's tokens; a target's logit.
template <class T, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head_stats_kernel(Operand weight, Operand hidden, int planes, int steps, int v0, int tiles_m, int tiles_n, HeadMask mask,
                                                                    const int32_t *count, const int32_t *row_of, const int32_t *target_of, float2 *parts, int parts_stride,
                                                                    float *target_logit) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int m, n;
    tile_of_block(blockIdx.x, tiles_m, tiles_n, m, n);
    const int rows = *count;
    if (n * Tile::kN >= rows) return;
    Tile tile;
    tile.run(weight, hidden, m * Tile::kM, n * Tile::kN, planes, 0, steps, lds);
    constexpr int kSpan = Tile::kMi * 16;                                 // tokens of a wave's share
    const int wave_m = Tile::wave() / Tile::kWavesN, from = v0 + m * Tile::kM + wave_m * kSpan, quad = Tile::lane() / 16;
    float2 *out = parts + (size_t)((v0 / Tile::kM + m) * Tile::kWavesM + wave_m) * parts_stride;
#pragma unroll
    for (int j = 0; j < Tile::kNj; ++j) {
        const int at = n * Tile::kN + Tile::n_of(j);
        const bool there = at < rows;
        uint32_t allowed[kSpan / 32];
        allowed_words<kSpan / 32>(mask, row_of, there ? at : rows - 1, from, allowed);
        const int target = target_of[there ? at : rows - 1] - from;       // within the share: whose logit is wanted
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < Tile::kMi; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int v = i * 16 + quad * 4 + e;
                if (v == target && there) target_logit[at] = tile.acc[i][j][e];
                if (!(allowed[i / 2] >> (i % 2 * 16 + quad * 4 + e) & 1u)) tile.acc[i][j][e] = -INFINITY;
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
        if (quad == 0 && there) out[at] = make_float2(top, sum);
    }
}

// A wave for every row: its parts joined, in 64 bits.
__global__ __launch_bounds__(256) void head_join_kernel(const int32_t *place, int rows, const float2 *parts, int parts_stride, int n_parts, const float *target_logit,
                                                        float *loss, float2 *stats) {
    const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (r >= rows) return;
    const int at = place[r];
    if (at < 0) {
        if (lane == 0) {
            if (loss) loss[r] = 0.0f;
            if (stats) stats[r] = make_float2(0.0f, 1.0f);
        }
        return;
    }
    float top = -INFINITY;
    for (int i = lane; i < n_parts; i += 64) top = fmaxf(top, parts[(size_t)i * parts_stride + at].x);
    top = wave_max(top);
    double sum = 0.0;
    for (int i = lane; i < n_parts; i += 64) {
        const float2 p = parts[(size_t)i * parts_stride + at];
        if (p.x > -INFINITY || p.y != p.y) sum += (double)p.y * exp((double)p.x - (double)top);
    }
    sum = wave_sum(sum);
    if (lane == 0) {
        if (loss) loss[r] = (float)(log(sum) + ((double)top - (double)target_logit[at]));
        if (stats) stats[r] = make_float2(top, (float)sum);
    }
}

// Two neighbouring 16-byte pieces of a row of the block's tile of slopes, kM tokens a row, are exchanged by the row's number: rows written side
// by side, and every eighth row read, lie on different banks.
__device__ __forceinline__ int slope_piece(int n, int piece) { return piece ^ ((n ^ (n >> 3)) & 15); }

// d weight takes the rows in steps of so many: up to the next multiple there are slopes, zeros behind the last row.
constexpr int kStepRows = kStepBytes / 2;

// The slopes of a piece of the vocabulary, in the operands' type: [row][plane][token] and [token][plane][row].
template <class T, class F, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head_slopes_kernel(Operand weight, Operand hidden, int planes, int steps, int v0, int tiles_m, int tiles_n, HeadMask mask,
                                                                     Taught taught, const float2 *stats, char *by_row, int64_t by_row_stride, int by_row_plane,
                                                                     char *by_token, int64_t by_token_stride, int by_token_plane) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int m, n;
    tile_of_block(blockIdx.x, tiles_m, tiles_n, m, n);
    const int rows = *taught.count;
    if (n * Tile::kN >= (rows + kStepRows - 1) / kStepRows * kStepRows) return;
    Tile tile;
    tile.run(weight, hidden, m * Tile::kM, n * Tile::kN, planes, 0, steps, lds);
    constexpr int kSpan = Tile::kMi * 16;
    const int wave_m = Tile::wave() / Tile::kWavesN, from = v0 + m * Tile::kM + wave_m * kSpan, quad = Tile::lane() / 16;
    const float scale = taught.scale[0];
    constexpr int kRow = Tile::kM * 2;                                    // bytes of a tile's row in LDS
    // four tokens' parts in the present plane, into the tile; what is left of them
    auto lay = [&](int i, int j, Float4 &x) {
        const int row = Tile::n_of(j), v = Tile::m_of(i);
        const uint2 two = make_uint2(F::pair(x[0], x[1]), F::pair(x[2], x[3]));
        *reinterpret_cast<uint2 *>(lds + row * kRow + slope_piece(row, v >> 3) * 16 + (v & 4) * 2) = two;
        if (planes > 1) x -= Float4{F::value(two.x & 0xFFFFu), F::value(two.x >> 16), F::value(two.y & 0xFFFFu), F::value(two.y >> 16)};
    };
    __syncthreads();                                                      // (all waves have read the tile's operands)
#pragma unroll
    for (int j = 0; j < Tile::kNj; ++j) {
        const int at = n * Tile::kN + Tile::n_of(j);
        const bool there = at < rows;
        const int place = there ? at : rows - 1;
        uint32_t allowed[kSpan / 32];
        allowed_words<kSpan / 32>(mask, taught.row, place, from, allowed);
        const int target = there ? taught.target[place] - from - quad * 4 : -1;
        const float2 sum = stats[taught.row[place]];
        const float g = taught.weight[place] * scale, share = 1.0f / sum.y;
#pragma unroll
        for (int i = 0; i < Tile::kMi; ++i) {
            const uint32_t four = there ? allowed[i / 2] >> (i % 2 * 16 + quad * 4) : 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float p = __builtin_amdgcn_exp2f((tile.acc[i][j][e] - sum.x) * kLog2E) * share;
                if (target == i * 16 + e) p -= 1.0f;
                tile.acc[i][j][e] = four >> e & 1u ? p * g : 0.0f;
            }
            lay(i, j, tile.acc[i][j]);
        }
    }
    for (int plane = 0; plane < planes; ++plane) {
        if (plane) {
            __syncthreads();                                              // (the plane before has been read)
#pragma unroll
            for (int j = 0; j < Tile::kNj; ++j)
#pragma unroll
                for (int i = 0; i < Tile::kMi; ++i) lay(i, j, tile.acc[i][j]);
        }
        __syncthreads();
        if (by_row) {
            constexpr int kPieces = Tile::kM / 8;
            for (int p = threadIdx.x; p < Tile::kN * kPieces; p += Tile::kThreads) {
                const int row = p / kPieces, piece = p % kPieces;
                *reinterpret_cast<uint4 *>(by_row + (int64_t)(n * Tile::kN + row) * by_row_stride + (int64_t)plane * by_row_plane + (m * Tile::kM + piece * 8) * 2) =
                    *reinterpret_cast<const uint4 *>(lds + row * kRow + slope_piece(row, piece) * 16);
            }
        }
        if (by_token) {
            constexpr int kPieces = Tile::kN / 8;
            for (int p = threadIdx.x; p < Tile::kM * kPieces; p += Tile::kThreads) {
                const int v = p / kPieces, row = p % kPieces * 8;
                uint32_t h[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] = *reinterpret_cast<const uint16_t *>(lds + (row + e) * kRow + slope_piece(row + e, v >> 3) * 16 + (v & 7) * 2);
                *reinterpret_cast<uint4 *>(by_token + (int64_t)(m * Tile::kM + v) * by_token_stride + (int64_t)plane * by_token_plane + (n * Tile::kN + row) * 2) =
                    make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
            }
        }
    }
}

// d hidden of the taught rows, over a piece of the vocabulary: sums[split][row][dim], of which each split takes its share of the piece's steps.
template <class T, class Tile>
__global__ __launch_bounds__(Tile::kThreads) void head_hidden_grad_kernel(Operand weight_t, Operand slopes, int planes, int steps, int splits, int tiles_m, int tiles_n,
                                                                          const int32_t *count, float *sums, int sums_stride, int sums_rows, bool first) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int m, n;
    tile_of_block(blockIdx.x, tiles_m * splits, tiles_n, m, n);
    if (n * Tile::kN >= *count) return;
    const int split = m / tiles_m;
    m -= split * tiles_m;
    Tile tile;
    tile.run(weight_t, slopes, m * Tile::kM, n * Tile::kN, planes, (int)((int64_t)steps * split / splits), (int)((int64_t)steps * (split + 1) / splits), lds);
#pragma unroll
    for (int j = 0; j < Tile::kNj; ++j)
#pragma unroll
        for (int i = 0; i < Tile::kMi; ++i) {
            const int row = n * Tile::kN + Tile::n_of(j), d = m * Tile::kM + Tile::m_of(i);
            if (d >= sums_stride) continue;                               // (a multiple of four)
            Float4 *at = reinterpret_cast<Float4 *>(sums + ((size_t)split * sums_rows + row) * sums_stride + d);
            *at = first ? tile.acc[i][j] : *at + tile.acc[i][j];
        }
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
__global__ __launch_bounds__(Tile::kThreads) void head_weight_grad_kernel(Operand hidden_t, Operand slopes, int planes, int tiles_m, int tiles_n, const int32_t *count,
                                                                          const float *scale, int dim, int tokens, typename F::Stored *out, int64_t out_stride) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int m, n;
    tile_of_block(blockIdx.x, tiles_m, tiles_n, m, n);
    const int steps = (*count * 2 + kStepBytes - 1) / kStepBytes * (planes > 1 ? kPlanePairs : 1);
    Tile tile;
    tile.run(hidden_t, slopes, m * Tile::kM, n * Tile::kN, planes, 0, steps, lds);
    const float back = scale[1];
#pragma unroll
    for (int j = 0; j < Tile::kNj; ++j) {
        const int v = n * Tile::kN + Tile::n_of(j);
        if (v >= tokens) continue;
        typename F::Stored *row = out + v * out_stride;
#pragma unroll
        for (int i = 0; i < Tile::kMi; ++i) {
            const int d = m * Tile::kM + Tile::m_of(i);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (d + e < dim) row[d + e] = (typename F::Stored)F::pattern(tile.acc[i][j][e] * back);
        }
    }
}

template <class S>
__global__ __launch_bounds__(256) void zero_rows_kernel(S *at, int dim, int64_t stride) {
    for (int d = blockIdx.y * 256 + threadIdx.x; d < dim; d += gridDim.y * 256) at[blockIdx.x * stride + d] = 0;
}

// ------------------------------------------------------------------------------------------------- host

size_t up(size_t n, size_t to) { return (n + to - 1) / to * to; }

// Where everything lies in the workspace, and how the vocabulary is cut.
struct Plan {
    int planes, padded_rows, pieces, piece;              // tokens of a piece: a multiple of 256
    bool packs_weight;                                   // the weights' rows are not as the products read them
    int hidden_bytes;                                    // of a packed row's plane
    int n_tile;                                          // rows of a tile
    int splits, sums_stride;
    size_t count, scale, place, row, target, weight, target_logit, parts, packed_hidden, packed_weight, stats, slopes_by_row, slopes_by_token, weight_t, hidden_t, sums, bytes;
};
// A tile has 256 tokens in every form.
constexpr int kTileTokens = 256, kWavesOfTokens = 4;
constexpr size_t kPieceBytes = (size_t)1 << 30;

int tile_rows(int rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }

Plan plan_of(const HeadRows &h, bool grads) {
    Plan p{};
    p.planes = h.type == kLogitF32 ? 3 : 1;
    const size_t size = h.type == kLogitF32 ? 4 : 2;
    p.n_tile = tile_rows(h.rows);
    p.padded_rows = (int)up(h.rows, std::max(p.n_tile, kStepRows));
    p.hidden_bytes = (int)up((size_t)h.dim * 2, kStepBytes);
    p.packs_weight = p.planes > 1 || h.dim % 8 != 0 || (reinterpret_cast<uintptr_t>(h.weight) | (uintptr_t)(h.weight_stride * size)) % 16 != 0 || h.weight_stride >= 1 << 22;
    // what a token takes while its piece is worked on
    const size_t each = (p.packs_weight ? (size_t)p.planes * p.hidden_bytes : 0) + (grads ? (size_t)p.planes * 2 * (2 * (size_t)p.padded_rows + h.dim) : 0);
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
        p.slopes_by_row = take((size_t)p.padded_rows * p.planes * p.piece * 2);
        p.slopes_by_token = take((size_t)p.piece * p.planes * p.padded_rows * 2);
        p.weight_t = take((size_t)h.dim * p.planes * p.piece * 2);
        p.hidden_t = take((size_t)h.dim * p.planes * p.padded_rows * 2);
        // few tiles of d hidden: the piece's steps are split until every unit has a tile, of at least 16 steps
        const int tiles = (int)(up(h.dim, kTileTokens) / kTileTokens * (p.padded_rows / p.n_tile)), steps = p.piece * 2 / kStepBytes * (p.planes > 1 ? kPlanePairs : 1);
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

template <class Kernel, class... Args>
hipError_t launch_tiles(Kernel kernel, int blocks, int threads, int lds, hipStream_t stream, Args... args) {
    // (a launch may have more than 64 KiB of LDS once its kernel is told so, on every device)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), lds, stream, args...);
    return hipGetLastError();
}
// fn(a tile's type) for tiles of so many rows.
template <class T, class Fn>
hipError_t with_tile(int n_tile, Fn fn) {
    switch (n_tile) {
        case 32: return fn((ProductTile<T, 256, 32, 4, 1, 4> *)nullptr);
        case 64: return fn((ProductTile<T, 256, 64, 4, 1, 3> *)nullptr);
        case 128: return fn((ProductTile<T, 256, 128, 4, 1, 3> *)nullptr);
        default: return fn((ProductTile<T, 256, 256, 4, 2, 2> *)nullptr);
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
    const int pairs = p.planes > 1 ? kPlanePairs : 1, steps = p.hidden_bytes / kStepBytes * pairs, tiles_n = p.padded_rows / p.n_tile;
    if (!stats) stats = w.as<float>(p.stats);
    if (forward) {
        for (int v0 = 0; v0 < h.vocab; v0 += p.piece) {
            const Operand weight = weight_operand<F>(h, p, w, v0, stream, e);
            if (e != hipSuccess) return e;
            const int tiles_m = (weight.rows + kTileTokens - 1) / kTileTokens;
            e = with_tile<T>(p.n_tile, [&](auto *tile) {
                typedef std::remove_pointer_t<decltype(tile)> Tile;
                static_assert(Tile::kM == kTileTokens && Tile::kWavesM == kWavesOfTokens, "parts of a row");
                return launch_tiles(head_stats_kernel<T, Tile>, tiles_m * tiles_n, Tile::kThreads, Tile::kLdsBytes, stream, weight, hidden, p.planes, steps, v0, tiles_m, tiles_n, mask,
                                    (const int32_t *)taught.count, (const int32_t *)taught.row, (const int32_t *)taught.target, w.as<float2>(p.parts), p.padded_rows,
                                    w.as<float>(p.target_logit));
            });
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(head_join_kernel, dim3((h.rows + 3) / 4), dim3(256), 0, stream, taught.place, h.rows, w.as<float2>(p.parts), p.padded_rows,
                           (h.vocab + kTileTokens - 1) / kTileTokens * kWavesOfTokens, w.as<float>(p.target_logit), loss, reinterpret_cast<float2 *>(stats));
    }
    if (!backward) return hipGetLastError();
    const int rows_bytes = p.padded_rows * 2;
    if (grad_weight) {
        e = launch_pack_transposed<F>(hidden_rows, h.hidden_stride, taught.row, taught.count, h.rows, p.padded_rows, h.dim, w.as<char>(p.hidden_t), rows_bytes, stream);
        if (e != hipSuccess) return e;
    }
    for (int v0 = 0; v0 < h.vocab; v0 += p.piece) {
        const Operand weight = weight_operand<F>(h, p, w, v0, stream, e);
        if (e != hipSuccess) return e;
        const int tokens = weight.rows, tiles_m = (tokens + kTileTokens - 1) / kTileTokens, tiles_d = (h.dim + kTileTokens - 1) / kTileTokens;
        const int tokens_bytes = tiles_m * kTileTokens * 2;
        e = with_tile<T>(p.n_tile, [&](auto *tile) {
            typedef std::remove_pointer_t<decltype(tile)> Tile;
            return launch_tiles(head_slopes_kernel<T, std::conditional_t<sizeof(Stored) == 4, LogitsBf16, F>, Tile>, tiles_m * tiles_n, Tile::kThreads,
                                std::max(Tile::kLdsBytes, Tile::kM * Tile::kN * 2), stream, weight, hidden, p.planes, steps, v0, tiles_m, tiles_n, mask, taught,
                                reinterpret_cast<const float2 *>(stats), grad_hidden ? w.as<char>(p.slopes_by_row) : nullptr, (int64_t)p.planes * p.piece * 2, p.piece * 2,
                                grad_weight ? w.as<char>(p.slopes_by_token) : nullptr, (int64_t)p.planes * rows_bytes, rows_bytes);
        });
        if (e != hipSuccess) return e;
        if (grad_hidden) {
            const auto *from = static_cast<const Stored *>(h.weight) + (int64_t)v0 * h.weight_stride;
            e = launch_pack_transposed<F>(from, h.weight_stride, nullptr, nullptr, tokens, tiles_m * kTileTokens, h.dim, w.as<char>(p.weight_t), p.piece * 2, stream);
            if (e != hipSuccess) return e;
            const Operand weight_t{w.as<char>(p.weight_t), (int64_t)p.planes * p.piece * 2, h.dim, p.piece * 2}, by_row{w.as<char>(p.slopes_by_row), (int64_t)p.planes * p.piece * 2, p.padded_rows, p.piece * 2};
            e = with_tile<T>(p.n_tile, [&](auto *tile) {
                typedef std::remove_pointer_t<decltype(tile)> Tile;
                return launch_tiles(head_hidden_grad_kernel<T, Tile>, tiles_d * p.splits * tiles_n, Tile::kThreads, Tile::kLdsBytes, stream, weight_t, by_row, p.planes,
                                    tokens_bytes / kStepBytes * pairs, p.splits, tiles_d, tiles_n, (const int32_t *)taught.count, w.as<float>(p.sums), p.sums_stride, p.padded_rows, v0 == 0);
            });
            if (e != hipSuccess) return e;
        }
        if (grad_weight) {
            const Operand hidden_t{w.as<char>(p.hidden_t), (int64_t)p.planes * rows_bytes, h.dim, rows_bytes}, by_token{w.as<char>(p.slopes_by_token), (int64_t)p.planes * rows_bytes, tiles_m * kTileTokens, rows_bytes};
            typedef ProductTile<T, 256, 256, 4, 2, 2> Tile;
            e = launch_tiles(head_weight_grad_kernel<T, F, Tile>, tiles_d * tiles_m, Tile::kThreads, Tile::kLdsBytes, stream, hidden_t, by_token, p.planes, tiles_d, tiles_m,
                             (const int32_t *)taught.count, (const float *)taught.scale, h.dim, tokens, static_cast<Stored *>(grad_weight) + (int64_t)v0 * grad_weight_stride, grad_weight_stride);
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
