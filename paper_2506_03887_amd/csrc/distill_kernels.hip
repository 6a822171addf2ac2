// gfx950 kernels of the distillation loss: a student's logits against a teacher's k best logits, both under the token mask, and the
// gradient.  With z = logit / tau over the row's open tokens (allowed, not -inf), p = softmax(z), and q the softmax of the teacher's listed
// logits / tau over those of its tokens that are open in the student's row,
//     loss = tau^2 sum_j q_j (log q_j - log p_(id j)),      d loss / d logit_v = tau (p_v - sum of the q_j with id j = v).
// A row of which nothing is listed has no loss and no gradient.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "argmax.hpp"
#include "lanes.hpp"
#include "launch.hpp"
#include "rows.hpp"
#include "stream_access.hpp"

namespace pre3 {

namespace {

template <class F>
__device__ __forceinline__ void store_eight(const float x[8], typename F::Stored *row, int g) {
    char *at = reinterpret_cast<char *>(row) + (size_t)(uint32_t)g * sizeof(Eight<F>);
    if constexpr (sizeof(typename F::Stored) == 2) {
        stream_store(make_uint4(F::pair(x[0], x[1]), F::pair(x[2], x[3]), F::pair(x[4], x[5]), F::pair(x[6], x[7])), reinterpret_cast<uint16_t *>(at));
    } else {
        stream_store(make_uint4(F::pattern(x[0]), F::pattern(x[1]), F::pattern(x[2]), F::pattern(x[3])), reinterpret_cast<uint16_t *>(at));
        stream_store(make_uint4(F::pattern(x[4]), F::pattern(x[5]), F::pattern(x[6]), F::pattern(x[7])), reinterpret_cast<uint16_t *>(at + 16));
    }
}

// A row's list is wave 0's, four entries a lane (64 apart): the token (-1: no entry, or its token is not open), the teacher's logit and the
// student's, then q.
struct List {
    static constexpr int kPer = kDistillMax / 64;
    int id[kPer];
    float teacher[kPer], student[kPer];
    double q[kPer], log_q[kPer];
};
__device__ __forceinline__ float teacher_logit(const DistillTeacher &t, size_t at) {
    if (t.type == kLogitF32) return static_cast<const float *>(t.logits)[at];
    const uint16_t h = static_cast<const uint16_t *>(t.logits)[at];
    return t.type == kLogitBf16 ? LogitsBf16::value(h) : LogitsF16::value(h);
}
// The ids; whether there is one of a token at all (rows without are not read).
__device__ __forceinline__ bool list_ids(const DistillTeacher &t, int b, int vocab, int lane, List &e) {
    bool some = false;
#pragma unroll
    for (int i = 0; i < e.kPer; ++i) {
        const int j = i * 64 + lane;
        e.id[i] = j < t.k ? t.ids[(size_t)b * t.k + j] : -1;
    }
#pragma unroll
    for (int i = 0; i < e.kPer; ++i) {
        if (e.id[i] >= vocab) e.id[i] = -1;
        some |= e.id[i] >= 0;
    }
    return __any(some);
}
template <class F>
__device__ __forceinline__ void list_logits(const DistillTeacher &t, int b, const Row<F> &row, int lane, List &e) {
#pragma unroll
    for (int i = 0; i < e.kPer; ++i) {
        e.teacher[i] = e.student[i] = -INFINITY;
        if (e.id[i] >= 0 && row.allows(e.id[i])) {
            e.student[i] = row.value(e.id[i]);
            e.teacher[i] = teacher_logit(t, (size_t)b * t.k + i * 64 + lane);
        }
    }
}
// q in 64 bits; whether an entry is left.
__device__ __forceinline__ bool list_shares(double inv_tau, List &e) {
    bool some = false;
    float best = -INFINITY;
#pragma unroll
    for (int i = 0; i < e.kPer; ++i) {
        if (e.student[i] == -INFINITY || e.teacher[i] == -INFINITY) e.id[i] = -1;      // (a NaN stays, and comes out as one)
        some |= e.id[i] >= 0;
        if (e.id[i] >= 0) best = fmaxf(best, e.teacher[i]);
    }
    best = wave_max(best);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < e.kPer; ++i) {
        e.log_q[i] = ((double)e.teacher[i] - (double)best) * inv_tau;
        e.q[i] = 0.0;
        if (e.id[i] >= 0) e.q[i] = exp(e.log_q[i]);
        sum += e.q[i];
    }
    sum = wave_sum(sum);
    const double log_sum = log(sum);
#pragma unroll
    for (int i = 0; i < e.kPer; ++i) {
        e.log_q[i] -= log_sum;
        e.q[i] = e.id[i] >= 0 ? e.q[i] / sum : 0.0;
    }
    return __any(some);
}

// The maximum of a row's open logits and the sum of 2^((logit - maximum) * scale); sum 0: nothing is open.  A thread keeps both
// for what it has seen, and weighs the sum anew when the maximum rises; threads are joined in 64 bits, always in the same order.  The maximum
// passes over NaNs, the sum does not: a thread that has seen nothing but a NaN has the maximum -inf, and its sum counts.
// 32-bit logits of more than a wave's rows: what a thread has seen is kept in 64 bits, sixteen tokens' weights are added to it at once.  In 32
// bits the weights of a row's mass vanish one by one beside a large one (gradients of 256 x 128,256 6.7e-7 off, so 2.8e-7; 64 us a call, so 63).
// Sixteen bits of a gradient do not show it, and a wave's rows are short (at most 24 tokens a sum; 3,000 x 3,001 f32 21.0 us, 22.0 in 64 bits).
struct Sum { float top; double z; };
__device__ __forceinline__ Sum joined_by_wave(float top, double z, float scale) {
    const float all = wave_max(top);
    return {all, wave_sum(z == 0.0 ? 0.0 : z * (double)__builtin_amdgcn_exp2f((top - all) * scale))};
}
template <int kBlock, class F, class Go>
__device__ __forceinline__ Sum sum_of(const Row<F> &row, int from, int to, float scale, const uint2 *table, Sum *s_sums, int tid, Go go) {
    constexpr int kU = kUnroll;
    constexpr bool kWide = sizeof(typename F::Stored) == 4 && kBlock > 64;
    float top = -INFINITY, z[4] = {};
    double before = 0.0;                       // kWide: what is not in z
    auto add = [&](const float *x, int n, float largest) {
        if (largest > top) {
            const float down = __builtin_amdgcn_exp2f((top - largest) * scale);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[i] *= down;
            if (kWide) before *= (double)down;
            top = largest;
        }
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int i = 0; i < n; ++i) z[i & 3] += __builtin_amdgcn_exp2f((x[i] - base) * scale);
        if (kWide) {
            before += (double)((z[0] + z[1]) + (z[2] + z[3]));
            z[0] = z[1] = z[2] = z[3] = 0.0f;
        }
    };
    const int whole = row.vocab >> 3;
    each_group<kBlock, F, false>(row, from, min(to, whole), tid, go, [&](int, const Eight<F> *e, const uint32_t *m) {
        float x[8 * kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) values_of<F>(e[u], m[u], table, x + 8 * u);
        float largest = x[0];
#pragma unroll
        for (int i = 1; i < 8 * kU; ++i) largest = fmaxf(largest, x[i]);
        add(x, 8 * kU, largest);
    });
    const int t = whole * 8 + tid;
    if (to > whole && t < row.vocab && row.allows(t)) {
        const float x = row.value(t);
        add(&x, 1, x);
    }
    const Sum wave = joined_by_wave(top, before + (double)((z[0] + z[1]) + (z[2] + z[3])), scale);
    if (kBlock == 64) return wave;
    if ((tid & 63) == 0) s_sums[tid >> 6] = wave;
    lds_barrier();
    const int at = tid & 63;
    const Sum other = at < kBlock / 64 ? s_sums[at] : Sum{-INFINITY, 0.0};
    return joined_by_wave(other.top, other.z, scale);
}

// The loss of a row, by wave 0.
__device__ __forceinline__ double loss_of(const List &e, const Sum &sum, double tau, double inv_tau) {
    const double log_z = log(sum.z);
    double term = 0.0;
#pragma unroll
    for (int i = 0; i < e.kPer; ++i)
        if (e.q[i] > 0.0 || e.q[i] != e.q[i]) term += e.q[i] * (e.log_q[i] - (((double)e.student[i] - (double)sum.top) * inv_tau - log_z));
    return tau * tau * wave_sum(term);
}

// The gradient of the groups `from` .. `to`: weight * (p - q).  A token that is not open has 2^-inf = 0 of the share; where the share is no
// number to multiply a zero with (a NaN or +inf in the row, an infinite weight, a quotient beyond 32 bits), the product is taken in 64 bits
// and such a token is told by its logit, in a loop of its own.
template <int kBlock, class F, class Go>
__device__ __forceinline__ void put_shares(const Row<F> &row, int from, int to, float top, float z, double weight, float scale, const uint2 *table, typename F::Stored *out,
                                           int tid, Go go) {
    constexpr int kU = kUnroll;
    const int whole = row.vocab >> 3, last = min(to, whole), t = whole * 8 + tid;
    const float share = (float)(weight / (double)z);
    const bool odd = __builtin_amdgcn_readfirstlane(!(fabsf(share) < INFINITY));          // (the same in every lane)
    auto odd_one = [&](float x) { return x == -INFINITY ? 0.0f : (float)((double)__builtin_amdgcn_exp2f((x - top) * scale) * (weight / (double)z)); };
    each_group<kBlock, F, true>(row, from, odd ? from : last, tid, go, [&](int g, const Eight<F> *eight, const uint32_t *m) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            float x[8];
            values_of<F>(eight[u], m[u], table, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f((x[i] - top) * scale) * share;
            if (g + u * kBlock < last) store_eight<F>(x, out, g + u * kBlock);
        }
    });
    if (odd) {
        for (int i = from * 8 + tid; i < last * 8; i += kBlock) out[i] = (typename F::Stored)F::pattern(row.allows(i) ? odd_one(row.value(i)) : 0.0f);
    }
    if (to > whole && t < row.vocab) {
        const float x = row.allows(t) ? row.value(t) : -INFINITY;
        out[t] = (typename F::Stored)F::pattern(odd ? odd_one(x) : __builtin_amdgcn_exp2f((x - top) * scale) * share);
    }
}
template <int kBlock, class F>
__device__ __forceinline__ void put_zeros(int from, int to, int vocab, typename F::Stored *out, int tid) {
    const int whole = vocab >> 3, last = min(to, whole), t = whole * 8 + tid;
    const float none[8] = {};
    for (int g = from + tid; g < last; g += kBlock) store_eight<F>(none, out, g);
    if (to > whole && t < vocab) out[t] = 0;
}
// The listed tokens, whole, over what put_shares has stored: p - q, which may be small beside both, is rounded once.  By the block;
// the work is wave 0's.
template <class F>
__device__ __forceinline__ void put_listed(const List &e, int k, int from, int to, int vocab, float top, double z, double weight, double inv_tau, int *s_id, double *s_q,
                                           typename F::Stored *out, int tid) {
    __builtin_amdgcn_s_waitcnt(0);             // the row's stores have arrived before these overwrite some of them
    __syncthreads();
    if (tid >= 64) return;
#pragma unroll
    for (int i = 0; i < e.kPer; ++i) { s_id[i * 64 + tid] = e.id[i]; s_q[i * 64 + tid] = e.q[i]; }
    wave_exchange();
#pragma unroll
    for (int i = 0; i < e.kPer; ++i) {
        const int at = i * 64 + tid, id = e.id[i];
        if (id < from * 8 || id >= min(to * 8, vocab)) continue;
        double q = 0.0;
        bool first = true;                     // of the entries with this token
        for (int j = 0; j < k; ++j) {
            if (s_id[j] != id) continue;
            q += s_q[j];
            if (j < at) first = false;
        }
        if (first) {
            const double p = exp(((double)e.student[i] - (double)top) * inv_tau) / z;      // (in 64 bits, like q: the largest gradients are these)
            out[id] = (typename F::Stored)F::pattern((float)((p - q) * weight));
        }
    }
}

struct DistillArgs {
    int vocab, n_words;
    int64_t row_stride;
    DistillTeacher teacher;
    float scale;                               // log2(e) / tau
    double inv_tau, tau;
    const float *row_weight;
    int64_t weight_stride, grad_stride;
    int segment;                               // groups of a block, where a row is several blocks'
};
template <class F>
__device__ __forceinline__ Row<F> row_of(const typename F::Stored *logits, const uint32_t *bitmask, const DistillArgs &a, int b) {
    return {logits + (size_t)b * a.row_stride, bitmask ? bitmask + (size_t)b * a.n_words : nullptr, a.vocab};
}
__device__ __forceinline__ double weight_of_row(const DistillArgs &a, int b) {
    return a.tau * (a.row_weight ? (double)a.row_weight[(size_t)b * a.weight_stride] : 1.0);
}

// The sums that the forward pass leaves of a row: a sum of 0 says that the row has no loss.  The sum is rounded to 32 bits, half a step of which a
// gradient of 32 bits may be off by for it; where loss and gradient are one pass it is rounded the same, so that both ways give the same.
__device__ __forceinline__ float2 stats_of(bool live, const Sum &sum) { return live ? make_float2(sum.top, (float)sum.z) : make_float2(0.0f, 0.0f); }

// One block a row: the loss, and with kGrad the gradient, for which the row is read again (from the caches, mostly: the rows of all
// blocks at a time are less than what the last one holds).
// Bound by HBM: loss and gradient of 4,096 x 128,256 bf16 move 2.55 GB (1.49 read, for 1.12 of logits and mask) in 412 us back to back in a
// graph, 6.2 TB/s, and in 413 to 449 launch by launch under a profiler, 6.0 in the mean; 256 x 128,256 f32, one row a unit, 0.30 GB in
// 62 us, 4.8 TB/s; the loss alone of 2,048 x 32,000 0.11 GB in 27 us, 4.0 TB/s.
template <int kBlock, class F, bool kGrad>
__global__ __launch_bounds__(kBlock) __attribute__((amdgpu_waves_per_eu(6))) void distill_row_kernel(const typename F::Stored *logits, const uint32_t *__restrict__ bitmask,
                                                                                                    DistillArgs a, float *__restrict__ loss, float2 *__restrict__ stats,
                                                                                                    typename F::Stored *grad) {
    __shared__ Sum s_sums[kBlock / 64];
    __shared__ uint2 s_table[16];
    __shared__ int s_id[kGrad ? kDistillMax : 1], s_live;
    __shared__ double s_q[kGrad ? kDistillMax : 1];
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.x, groups = (a.vocab + 7) >> 3;
    const bool lists = __builtin_amdgcn_readfirstlane(tid >> 6) == 0;
    const Row<F> row = row_of<F>(logits, bitmask, a, b);
    List e;
    bool live = true;
    mask_nibble_table_init(s_table, tid);
    const Sum sum = sum_of<kBlock, F>(row, 0, groups, a.scale, s_table, s_sums, tid, [&]() {
        if (lists) {
            const bool some = list_ids(a.teacher, b, a.vocab, lane, e);
            if (lane == 0) s_live = some;
        }
        lds_barrier();
        live = s_live;
        if (lists && live) list_logits<F>(a.teacher, b, row, lane, e);
        return live;
    });
    if (lists) {
        double value = 0.0;
        if (live) live = list_shares(a.inv_tau, e);
        if (live) value = loss_of(e, sum, a.tau, a.inv_tau);
        if (lane == 0) {
            loss[b] = (float)value;
            if (stats) stats[b] = stats_of(live, sum);
            s_live = live;
        }
    }
    if (!kGrad) return;
    lds_barrier();
    typename F::Stored *out = grad + (size_t)b * a.grad_stride;
    if (!s_live) {
        put_zeros<kBlock, F>(0, groups, a.vocab, out, tid);
        return;
    }
    const double weight = weight_of_row(a, b);
    const float z = (float)sum.z;
    put_shares<kBlock, F>(row, 0, groups, sum.top, z, weight, a.scale, s_table, out, tid, []() { return true; });
    put_listed<F>(e, a.teacher.k, 0, groups, a.vocab, sum.top, (double)z, weight, a.inv_tau, s_id, s_q, out, tid);
}

// The gradient alone, from the sums that the forward pass has left; a row may be several blocks' (the grid's second dimension, which
// ends at 65,535: the rows are the first one).  Bound by HBM: 2,048 x 32,000 45 us, 5.3 TB/s.
template <int kBlock, class F>
__global__ __launch_bounds__(kBlock) __attribute__((amdgpu_waves_per_eu(6))) void distill_grad_kernel(const typename F::Stored *logits, const uint32_t *__restrict__ bitmask,
                                                                                                     DistillArgs a, const float2 *__restrict__ stats,
                                                                                                     typename F::Stored *grad) {
    __shared__ uint2 s_table[16];
    __shared__ int s_id[kDistillMax];
    __shared__ double s_q[kDistillMax];
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.x, from = blockIdx.y * a.segment, groups = (a.vocab + 7) >> 3, to = min(from + a.segment, groups);
    const bool lists = __builtin_amdgcn_readfirstlane(tid >> 6) == 0;
    const Row<F> row = row_of<F>(logits, bitmask, a, b);
    typename F::Stored *out = grad + (size_t)b * a.grad_stride;
    const float2 st = stats[b];
    if (st.y == 0.0f) {
        put_zeros<kBlock, F>(from, to, a.vocab, out, tid);
        return;
    }
    const double weight = weight_of_row(a, b);
    List e;
    mask_nibble_table_init(s_table, tid);
    put_shares<kBlock, F>(row, from, to, st.x, st.y, weight, a.scale, s_table, out, tid, [&]() {
        if (lists) {                           // (before the first store: the gradient may take the logits' place)
            list_ids(a.teacher, b, a.vocab, lane, e);
            list_logits<F>(a.teacher, b, row, lane, e);
            list_shares(a.inv_tau, e);
        }
        lds_barrier();
        return true;
    });
    put_listed<F>(e, a.teacher.k, from, to, a.vocab, st.x, (double)st.y, weight, a.inv_tau, s_id, s_q, out, tid);
}

// Few long rows: the sums of a row's segments by a block each, then joined by a wave a row.  (96 x 100,003 f16: 7.0 + 3.6 us.)
template <int kBlock, class F>
__global__ __launch_bounds__(kBlock) __attribute__((amdgpu_waves_per_eu(6))) void distill_part_kernel(const typename F::Stored *__restrict__ logits,
                                                                                                     const uint32_t *__restrict__ bitmask, DistillArgs a,
                                                                                                     float2 *__restrict__ parts) {
    __shared__ Sum s_sums[kBlock / 64];
    __shared__ uint2 s_table[16];
    __shared__ int s_live;
    const int tid = threadIdx.x, b = blockIdx.x, from = blockIdx.y * a.segment, groups = (a.vocab + 7) >> 3;
    mask_nibble_table_init(s_table, tid);
    bool live = true;
    const Sum sum = sum_of<kBlock, F>(row_of<F>(logits, bitmask, a, b), from, min(from + a.segment, groups), a.scale, s_table, s_sums, tid, [&]() {
        if (tid < 64) {
            List e;
            const bool some = list_ids(a.teacher, b, a.vocab, tid, e);
            if (tid == 0) s_live = some;
        }
        lds_barrier();
        live = s_live;
        return live;
    });
    if (tid == 0 && live) parts[(size_t)b * gridDim.y + blockIdx.y] = make_float2(sum.top, (float)sum.z);
}
constexpr int kMostParts = 64;
template <class F>
__global__ __launch_bounds__(64) void distill_join_kernel(const typename F::Stored *__restrict__ logits, const uint32_t *__restrict__ bitmask, DistillArgs a,
                                                         const float2 *__restrict__ parts, int n_parts, float *__restrict__ loss, float2 *__restrict__ stats) {
    const int lane = threadIdx.x, b = blockIdx.x;
    const Row<F> row = row_of<F>(logits, bitmask, a, b);
    const float2 part = lane < n_parts ? parts[(size_t)b * n_parts + lane] : make_float2(-INFINITY, 0.0f);
    List e;
    Sum sum = {0.0f, 0.0};
    double value = 0.0;
    bool live = list_ids(a.teacher, b, a.vocab, lane, e);
    if (live) {
        list_logits<F>(a.teacher, b, row, lane, e);
        live = list_shares(a.inv_tau, e);
    }
    if (live) {                                // (else the parts may not have been written)
        sum = joined_by_wave(part.x, (double)part.y, a.scale);
        value = loss_of(e, sum, a.tau, a.inv_tau);
    }
    if (lane == 0) {
        loss[b] = (float)value;
        if (stats) stats[b] = stats_of(live, sum);
    }
}

template <int kBlock, class F>
void launch_forward(const DistillRows &r, DistillArgs a, int segments, float *loss, float2 *stats, float2 *parts, typename F::Stored *grad, hipStream_t stream) {
    const auto *logits = static_cast<const typename F::Stored *>(r.logits);
    if (segments > 1) {
        a.segment = ((r.vocab + 7) / 8 + segments - 1) / segments;
        hipLaunchKernelGGL((distill_part_kernel<kBlock, F>), dim3(r.rows, segments), dim3(kBlock), 0, stream, logits, r.bitmask, a, parts);
        hipLaunchKernelGGL((distill_join_kernel<F>), dim3(r.rows), dim3(64), 0, stream, logits, r.bitmask, a, parts, segments, loss, stats);
    } else if (grad) {
        hipLaunchKernelGGL((distill_row_kernel<kBlock, F, true>), dim3(r.rows), dim3(kBlock), 0, stream, logits, r.bitmask, a, loss, stats, grad);
    } else {
        hipLaunchKernelGGL((distill_row_kernel<kBlock, F, false>), dim3(r.rows), dim3(kBlock), 0, stream, logits, r.bitmask, a, loss, stats, grad);
    }
}
template <int kBlock, class F>
void launch_grad(const DistillRows &r, DistillArgs a, int segments, const float2 *stats, typename F::Stored *grad, hipStream_t stream) {
    a.segment = ((r.vocab + 7) / 8 + segments - 1) / segments;
    hipLaunchKernelGGL((distill_grad_kernel<kBlock, F>), dim3(r.rows, segments), dim3(kBlock), 0, stream, static_cast<const typename F::Stored *>(r.logits), r.bitmask, a,
                       stats, grad);
}
// fn(threads of a block) for so many blocks of so many tokens.  us a call, loss and gradient at once unless it says otherwise:
// * one wave up to 1,024 tokens (2,000 x 1,000: 10.9, with 256 threads 14.5), and up to 6,144 where six or more share a unit (3,000 x
//   3,000 18.7 and 22.7, f32 21.8 and 25.5; 3,000 x 6,500 f32 44.8 and 41.4; 256 x 5,000 12.8 and 10.3, 1,400 x 5,000 17.4 and 17.9);
// * 512 threads where a row's loads are what a block waits for: 32-bit rows beyond 16,384 tokens (1,500 x 24,000 63.0, with 256 threads 71.1),
//   16-bit rows beyond 56,000 (2,000 x 60,000 114.7 and 126.3) and, of few rows, beyond 28,000 (500 x 60,000 36.1 and 42.6, 500 x 30,000 in
//   two calls 25.4 and 27.6; but 1,500 x 32,000 in two calls 58.6 and 56.7);
// * 1,024 for the longest, since one block's waves then fill a unit: 16-bit rows beyond 80,000 (200 x 100,000 30.0, with 512 threads 33.7; 2,000 x
//   150,000 259.9 and 273.3; 500 x 70,000 38.4 and 39.0), in two calls of few rows only (200 x 100,000 33.2 and 37.4, 1,000 x 100,000 119.4 and 114.3);
//   32-bit ones beyond 28,000, in two calls beyond 56,000, of more than 256 rows (700 x 30,000 41.3 and 46.3, 700 x 128,256 159.3 and 187.3, in two
//   calls 181.8 and 192.7, 700 x 30,000 55.0 and 53.0; 200 x 128,256 59.0 and 57.2);
// * 256 in between.
template <class Fn>
void with_block(int rows, int tokens, int bytes, bool at_once, Fn fn) {
    const bool longest = bytes == 4 ? rows > 256 && tokens > (at_once ? 28000 : 56000) : tokens > 80000 && (at_once || rows <= 768);
    if (tokens <= 1024 || (tokens <= 6144 && rows >= 1536)) fn(std::integral_constant<int, 64>());
    else if (longest) fn(std::integral_constant<int, 1024>());
    else if (tokens <= (bytes == 4 ? 16384 : rows <= 768 ? 28000 : 56000)) fn(std::integral_constant<int, 256>());
    else fn(std::integral_constant<int, 512>());
}

template <class F>
hipError_t launch(const DistillRows &r, const DistillTeacher &teacher, double tau, bool forward, const float *row_weight, int64_t weight_stride, float *loss,
                  float *stats, void *workspace, void *grad, int64_t grad_stride, hipStream_t stream) {
    DistillArgs a{};
    a.vocab = r.vocab;
    a.n_words = (r.vocab + 31) / 32;
    a.row_stride = r.row_stride;
    a.teacher = teacher;
    a.inv_tau = 1.0 / tau;
    a.tau = tau;
    a.scale = (float)(1.44269504088896340736 * a.inv_tau);
    a.row_weight = row_weight;
    a.weight_stride = weight_stride;
    a.grad_stride = grad_stride;
    auto *out = static_cast<typename F::Stored *>(grad);
    auto *sums = reinterpret_cast<float2 *>(stats), *parts = static_cast<float2 *>(workspace);
    // (loss and gradient at once by one block read the row from memory once: several blocks and a second launch gain beyond 36,864 tokens,
    // 24 x 65,536 23.8 and 14.4 us, 96 x 32,000 16.7 and 17.2, 64 x 17,000 13.0 and 15.9)
    const int most = distill_segments(r.rows, r.vocab), segments = workspace && (!(forward && grad) || r.vocab > 36864) ? most : 1;
    if (forward) {
        // workspace: the sums of a row's blocks, behind the rows' own where the caller does not want them
        if (!sums && segments > 1) { sums = parts; parts += r.rows; }
        with_block(r.rows * segments, (r.vocab + segments - 1) / segments, sizeof(typename F::Stored), grad != nullptr, [&](auto block) { launch_forward<decltype(block)::value, F>(r, a, segments, loss, sums, parts, out, stream); });
        if (segments == 1) return hipGetLastError();
    }
    if (grad) {
        // the blocks of a row read its listed logits: where the gradient overwrites them, one block has the row to itself
        const int blocks = grad == r.logits ? 1 : most;
        with_block(r.rows * blocks, (r.vocab + blocks - 1) / blocks, sizeof(typename F::Stored), false, [&](auto block) { launch_grad<decltype(block)::value, F>(r, a, blocks, sums, out, stream); });
    }
    return hipGetLastError();
}

}  // namespace

// Few long rows go over several blocks each, of at least 8,192 tokens, two blocks to a unit.  Loss and gradient through a kept sum, one block a
// row and several: 24 x 65,536 26.7 and 14.7 us, 96 x 32,000 19.4 and 17.3, 128 x 128,256 37.4 and 30.4; 192 x 128,256 43.4 and 46.7, 64 x 17,000
// 16.2 and 16.4.
int distill_segments(int rows, int vocab) {
    constexpr int kBlocks = 512, kSegmentTokens = 8192, kMostRows = 160, kLeastTokens = 24576;
    if (rows < 1 || rows > kMostRows || vocab < kLeastTokens) return 1;
    const int most = vocab / kSegmentTokens < kMostParts ? vocab / kSegmentTokens : kMostParts;
    return most < kBlocks / rows ? most : kBlocks / rows;
}
size_t distill_workspace_bytes(int rows, int vocab) {
    const int segments = distill_segments(rows, vocab);
    return rows < 1 || segments < 2 ? 0 : (size_t)rows * (segments + 1) * sizeof(float2);
}

hipError_t launch_distill(const DistillRows &rows, const DistillTeacher &teacher, double tau, bool forward, const float *row_weight, int64_t weight_stride, float *loss,
                          float *stats, void *workspace, void *grad, int64_t grad_stride, hipStream_t stream) {
    if (rows.rows == 0 || rows.vocab == 0) return hipSuccess;
    switch (rows.type) {
        case kLogitBf16: return launch<LogitsBf16>(rows, teacher, tau, forward, row_weight, weight_stride, loss, stats, workspace, grad, grad_stride, stream);
        case kLogitF16: return launch<LogitsF16>(rows, teacher, tau, forward, row_weight, weight_stride, loss, stats, workspace, grad, grad_stride, stream);
        default: return launch<LogitsF32>(rows, teacher, tau, forward, row_weight, weight_stride, loss, stats, workspace, grad, grad_stride, stream);
    }
}

}  // namespace pre3
