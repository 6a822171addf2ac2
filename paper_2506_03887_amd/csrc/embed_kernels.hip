// gfx950 kernels of the table that tokens are looked up in: rows of it by token, times a scale, and its gradient,
//     out_i = scale * table[t_i]   (zeros where t_i is no token),      d table[v] = scale * sum over the i with t_i = v of d out_i.
// The gradient's sums run over the tokens in the order of their ids, equal ones in the order of their places, so that every row of it is
// summed in one order and written once, without atomics.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "launch.hpp"
#include "pack.hpp"
#include "rows.hpp"

namespace pre3 {

namespace {

__device__ __forceinline__ int64_t id_at(const void *ids, int bytes, int64_t i) {
    return bytes == 8 ? static_cast<const int64_t *>(ids)[i] : static_cast<const int32_t *>(ids)[i];
}
// A wave for 2,048 numbers of a row, 32 a lane, all of them on their way at once.
constexpr int kWaveNumbers = 2048;
template <class F>
__global__ __launch_bounds__(64) void embed_kernel(const typename F::Stored *table, int64_t table_stride, const void *ids, int id_bytes, int vocab, int dim, float scale,
                                                   typename F::Stored *out, int64_t out_stride) {
    const int i = blockIdx.x, first = blockIdx.y * kWaveNumbers + threadIdx.x * 8;
    const int64_t t = id_at(ids, id_bytes, i);
    const bool is = t >= 0 && t < vocab;
    const auto *row = table + (is ? t : 0) * table_stride;
    float x[4][8];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int at = first + g * 512;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[g][e] = 0.0f;
        if (is && at < dim) eight_of<F>(row, at, dim, x[g]);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int at = first + g * 512;
        if (at >= dim) break;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[g][e] = is ? x[g][e] * scale : 0.0f;
        put_eight<F, true>(x[g], out + i * out_stride, at, dim);
    }
}

// ---- tokens in the order of their ids.  First the 512 of a block, each at the number of those that lie before it; then over all blocks: where a
// token lies among another block's 512 a bisection tells.
constexpr int kSorted = 512;
constexpr int kSlab = 16;                       // blocks' lists in LDS at a time
constexpr uint32_t kNoKey = 0x7FFFFFFFu;        // behind the last token

// Blocks beyond the sort's write zeros, all over the gradient: they have something to do while the few blocks of the sort are busy.
// (1 GiB by blocks that write 8 KiB, 16 bytes a thread: 6.4 TB/s; four times 16 bytes a thread 5.7, in a loop by 4,096 blocks 5.0)
constexpr int kZeros = kSorted * 16;
__device__ __forceinline__ void zeros(char *at, int64_t bytes, int64_t block) {
    const int64_t i = block * kZeros + threadIdx.x * 16;
    if (i + 16 <= bytes) stream_store(make_uint4(0, 0, 0, 0), reinterpret_cast<uint16_t *>(at + i));
    else
        for (int64_t b = i; b < bytes; b += 2) *reinterpret_cast<uint16_t *>(at + b) = 0;
}
// ids that are no token get the key `vocab`, behind all tokens.
__global__ __launch_bounds__(kSorted) void embed_sort_kernel(const void *ids, int id_bytes, int n, int vocab, int lists, uint32_t *keys, int32_t *places, char *grad, int64_t grad_bytes) {
    if ((int)blockIdx.x >= lists) return zeros(grad, grad_bytes, blockIdx.x - lists);
    __shared__ __attribute__((aligned(16))) uint32_t all[kSorted];
    const int tid = threadIdx.x, i = blockIdx.x * kSorted + tid;
    uint32_t key = kNoKey;
    if (i < n) {
        const int64_t t = id_at(ids, id_bytes, i);
        key = t >= 0 && t < vocab ? (uint32_t)t : (uint32_t)vocab;
    }
    const uint32_t mine = min(key, 0x7FFFFFu) << 9 | (uint32_t)tid;       // all of them differ
    all[tid] = mine;
    __syncthreads();
    int at = 0;
    for (int j = 0; j < kSorted; j += 4) {
        const uint4 four = *reinterpret_cast<const uint4 *>(&all[j]);
        at += (four.x < mine) + (four.y < mine) + (four.z < mine) + (four.w < mine);
    }
    keys[blockIdx.x * kSorted + at] = key;
    places[blockIdx.x * kSorted + at] = i;
}
__global__ __launch_bounds__(kSorted) void embed_merge_kernel(const uint32_t *keys, const int32_t *places, int n, int lists, uint32_t *sorted_keys, int32_t *sorted_places, char *grad,
                                                              int64_t grad_bytes) {
    if ((int)blockIdx.x >= lists) return zeros(grad, grad_bytes, blockIdx.x - lists);
    __shared__ uint32_t slab[kSlab][kSorted];
    const int tid = threadIdx.x, mine = blockIdx.x;
    const uint32_t key = keys[mine * kSorted + tid];
    int at = 0;
    for (int l0 = 0; l0 < lists; l0 += kSlab) {
        __syncthreads();
#pragma unroll
        for (int l = 0; l < kSlab; ++l)
            if (l0 + l < lists) slab[l][tid] = keys[(l0 + l) * kSorted + tid];
        __syncthreads();
#pragma unroll
        for (int l = 0; l < kSlab; ++l) {
            if (l0 + l >= lists) break;
            // the number of keys below this one; of an earlier list, equal ones too
            const uint32_t limit = key + (l0 + l < mine ? 1u : 0u);
            int below = 0;
#pragma unroll
            for (int half = kSorted / 2; half > 0; half /= 2)
                if (slab[l][below + half - 1] < limit) below += half;
            if (slab[l][below] < limit) ++below;
            at += l0 + l == mine ? tid : below;
        }
    }
    const int place = places[mine * kSorted + tid];
    if (place < n) {
        sorted_keys[at] = key;
        sorted_places[at] = place;
    }
}

// ---- sums of the sorted places.  A wave takes a run of them, of up to 64, and 512 numbers of the rows, eight a lane; the next wave the next 512.  A
// token whose places lie within a run is written at once; else its part of the run goes to parts[run][0] (it began before the run) or [1]
// (it begins here and goes on).
constexpr int kMostRun = 64, kLeastRun = 8, kWaveColumns = 512, kAhead = 8;
template <class F>
__global__ __launch_bounds__(256) void embed_grad_kernel(const typename F::Stored *rows, int64_t row_stride, const uint32_t *keys, const int32_t *places, int n, int vocab, int dim, float scale,
                                                         int of_run, int columns, float *parts, int parts_stride, typename F::Stored *out, int64_t out_stride) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6))), lane = threadIdx.x & 63, run = wave / columns, first = run * of_run;
    if (first >= n) return;
    const int d = wave % columns * kWaveColumns + lane * 8, count = min(of_run, n - first);
    // lane i holds the run's i-th place; the keys on both sides
    const uint32_t key_of = lane < count ? keys[first + lane] : kNoKey;
    const int place_of = lane < count ? places[first + lane] : 0;
    const uint32_t before = first > 0 ? keys[first - 1] : kNoKey, behind = first + count < n ? keys[first + count] : kNoKey;
    float sum[8] = {};
    auto flush = [&](uint32_t key, bool began, bool goes_on) {
        if (d >= dim) return;
        if (!began && !goes_on) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = sum[e] * scale;
            put_eight<F, true>(y, out + (int64_t)key * out_stride, d, dim);
        } else {
            float *to = parts + ((size_t)run * 2 + (began ? 0 : 1)) * parts_stride + d;     // (a multiple of eight)
            *reinterpret_cast<float4 *>(to) = make_float4(sum[0], sum[1], sum[2], sum[3]);
            *reinterpret_cast<float4 *>(to + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
        }
    };
    uint32_t key = (uint32_t)__builtin_amdgcn_readlane((int)key_of, 0);
    bool began = key == before;
    for (int i0 = 0; i0 < count; i0 += kAhead) {
        float x[kAhead][8];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int place = __builtin_amdgcn_readlane(place_of, min(i0 + i, count - 1));
            if (d < dim) eight_of<F>(rows + place * row_stride, d, dim, x[i]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (i0 + i >= count) break;
            const uint32_t next = (uint32_t)__builtin_amdgcn_readlane((int)key_of, i0 + i);
            if (next != key) {
                if (key < (uint32_t)vocab) flush(key, began, false);
                key = next;
                began = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += x[i][e];
        }
    }
    if (key < (uint32_t)vocab) flush(key, began, key == behind);
}
// The tokens that go on from one run to the next: four waves add up every fourth of their parts, and the waves' sums are added in order.
template <class F>
__global__ __launch_bounds__(256) void embed_join_kernel(const uint32_t *keys, int n, int vocab, int dim, float scale, int of_run, const float *parts, int parts_stride,
                                                         typename F::Stored *out, int64_t out_stride) {
    __shared__ float sums[4][64][9];
    const int run = blockIdx.x, next = (run + 1) * of_run;                // there is one behind
    const uint32_t key = keys[next - 1];
    if (key >= (uint32_t)vocab || keys[next] != key) return;
    if (run > 0 && keys[run * of_run] == key && keys[run * of_run - 1] == key) return;      // it began before
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d = blockIdx.y * kWaveColumns + lane * 8;
    float sum[8] = {};
    if (d < dim) {
#pragma unroll 4
        for (int r = run + wave; r * of_run < n && (r == run || keys[r * of_run] == key); r += 4) {
            const float *from = parts + ((size_t)r * 2 + (r == run ? 1 : 0)) * parts_stride + d;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += from[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][lane][e] = sum[e];
    __syncthreads();
    if (wave || d >= dim) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = (((sum[e] + sums[1][lane][e]) + sums[2][lane][e]) + sums[3][lane][e]) * scale;
    put_eight<F, true>(sum, out + (int64_t)key * out_stride, d, dim);
}

size_t up(size_t n, size_t to) { return (n + to - 1) / to * to; }
struct EmbedPlan {
    int lists, run, columns, parts_stride;
    size_t keys, places, sorted_keys, sorted_places, parts, bytes;
};
EmbedPlan plan_of(int n, int dim) {
    EmbedPlan p{};
    p.lists = (n + kSorted - 1) / kSorted;
    p.parts_stride = (int)up(dim, 8);
    p.columns = (dim + kWaveColumns - 1) / kWaveColumns;
    // long runs have few parts to join, short ones give every unit's eight waves something to do
    p.run = kMostRun;
    while (p.run > kLeastRun && (int64_t)n * p.columns / p.run < 2048) p.run /= 2;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t from = at; at += up(bytes, 256); return from; };
    for (size_t *x : {&p.keys, &p.places, &p.sorted_keys, &p.sorted_places}) *x = take((size_t)p.lists * kSorted * 4);
    p.parts = take((size_t)((n + p.run - 1) / p.run) * 2 * p.parts_stride * 4);
    p.bytes = at;
    return p;
}

template <class F>
hipError_t embed(const EmbedRows &r, void *out, int64_t out_stride, hipStream_t stream) {
    typedef typename F::Stored Stored;
    hipLaunchKernelGGL((embed_kernel<F>), dim3(r.rows, (r.dim + kWaveNumbers - 1) / kWaveNumbers), dim3(64), 0, stream, static_cast<const Stored *>(r.table), r.table_stride, r.ids,
                       r.id_bytes, r.vocab, r.dim, r.scale, static_cast<Stored *>(out), out_stride);
    return hipGetLastError();
}
template <class F>
hipError_t grad(const EmbedRows &r, const void *rows_grad, int64_t rows_stride, void *out, void *workspace, hipStream_t stream) {
    typedef typename F::Stored Stored;
    const EmbedPlan p = plan_of(r.rows, r.dim);
    char *w = static_cast<char *>(workspace);
    auto *keys = reinterpret_cast<uint32_t *>(w + p.keys), *sorted_keys = reinterpret_cast<uint32_t *>(w + p.sorted_keys);
    auto *places = reinterpret_cast<int32_t *>(w + p.places), *sorted_places = reinterpret_cast<int32_t *>(w + p.sorted_places);
    auto *parts = reinterpret_cast<float *>(w + p.parts);
    auto *to = static_cast<Stored *>(out);
    const int64_t bytes = (int64_t)r.vocab * r.dim * sizeof(Stored);
    const bool merges = p.lists > 1;
    char *all = reinterpret_cast<char *>(out);
    const int64_t blocks = (bytes + kZeros - 1) / kZeros, now = merges ? blocks / 2 : blocks;       // half the zeros beside each
    hipLaunchKernelGGL(embed_sort_kernel, dim3((uint32_t)(p.lists + now)), dim3(kSorted), 0, stream, r.ids, r.id_bytes, r.rows, r.vocab, p.lists, merges ? keys : sorted_keys,
                       merges ? places : sorted_places, all, std::min(bytes, now * kZeros));
    if (merges)
        hipLaunchKernelGGL(embed_merge_kernel, dim3((uint32_t)(p.lists + blocks - now)), dim3(kSorted), 0, stream, keys, places, r.rows, p.lists, sorted_keys, sorted_places,
                           all + now * kZeros, bytes - now * kZeros);
    if (r.rows == 0) return hipGetLastError();
    const int runs = (r.rows + p.run - 1) / p.run;
    hipLaunchKernelGGL((embed_grad_kernel<F>), dim3((runs * p.columns + 3) / 4), dim3(256), 0, stream, static_cast<const Stored *>(rows_grad), rows_stride, sorted_keys, sorted_places, r.rows,
                       r.vocab, r.dim, r.scale, p.run, p.columns, parts, p.parts_stride, to, (int64_t)r.dim);
    if (runs > 1)
        hipLaunchKernelGGL((embed_join_kernel<F>), dim3(runs - 1, p.columns), dim3(256), 0, stream, sorted_keys, r.rows, r.vocab, r.dim, r.scale, p.run, parts, p.parts_stride, to,
                           (int64_t)r.dim);
    return hipGetLastError();
}

}  // namespace

size_t embed_workspace_bytes(int rows, int dim) { return plan_of(rows, dim).bytes; }
hipError_t launch_embed(const EmbedRows &r, void *out, int64_t out_stride, hipStream_t stream) {
    return r.type == kLogitBf16 ? embed<LogitsBf16>(r, out, out_stride, stream) : r.type == kLogitF16 ? embed<LogitsF16>(r, out, out_stride, stream) : embed<LogitsF32>(r, out, out_stride, stream);
}
hipError_t launch_embed_grad(const EmbedRows &r, const void *rows_grad, int64_t rows_stride, void *out, void *workspace, hipStream_t stream) {
    return r.type == kLogitBf16 ? grad<LogitsBf16>(r, rows_grad, rows_stride, out, workspace, stream)
           : r.type == kLogitF16 ? grad<LogitsF16>(r, rows_grad, rows_stride, out, workspace, stream) : grad<LogitsF32>(r, rows_grad, rows_stride, out, workspace, stream);
}

}  // namespace pre3
