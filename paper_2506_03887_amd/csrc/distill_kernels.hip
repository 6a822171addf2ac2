// gfx950 kernels of the distillation loss: a student's logits against a teacher's k best logits, both under the token mask, and the
// gradient.  With z = logit / tau over the row's open tokens (allowed, not -inf), p = softmax(z), and q the softmax of the teacher's listed
// logits / tau over those of its tokens that are open in the student's row,
//     loss = tau^2 sum_j q_j (log q_j - log p_(id j)),      d loss / d logit_v = tau (p_v - sum of the q_j with id j = v).
// A row of which nothing is listed has no loss and no gradient.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "launch.hpp"
#include "stream_access.hpp"

namespace pre3 {

namespace {

constexpr int kDistillBlock = 1024, kDistillWaves = kDistillBlock / 64;

// Logits of one type: eight of them as loaded, as numbers, and back.
struct DistillBf16 {
    typedef uint16_t Stored;
    __device__ static float value(uint32_t h) { return __uint_as_float(h << 16); }
    __device__ static uint32_t pattern(float x) {
        const __bf16 y = (__bf16)x;
        return __builtin_bit_cast(uint16_t, y);
    }
};
struct DistillF16 {
    typedef uint16_t Stored;
    __device__ static float value(uint32_t h) { return (float)__builtin_bit_cast(_Float16, (uint16_t)h); }
    __device__ static uint32_t pattern(float x) {
        const _Float16 y = (_Float16)x;
        return __builtin_bit_cast(uint16_t, y);
    }
};
struct DistillF32 {
    typedef uint32_t Stored;
    __device__ static float value(uint32_t h) { return __uint_as_float(h); }
    __device__ static uint32_t pattern(float x) { return __float_as_uint(x); }
};
template <class F>
__device__ __forceinline__ void load_eight(const typename F::Stored *p, float x[8]) {
    if constexpr (sizeof(typename F::Stored) == 2) {
        const uint4 v = stream_load(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = F::value(w[i] & 0xFFFFu); x[2 * i + 1] = F::value(w[i] >> 16); }
    } else {
        const uint4 v = stream_load(reinterpret_cast<const uint16_t *>(p)), w = stream_load(reinterpret_cast<const uint16_t *>(p + 4));
        const uint32_t y[8] = {v.x, v.y, v.z, v.w, w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = F::value(y[i]);
    }
}
template <class F>
__device__ __forceinline__ void store_eight(const float x[8], typename F::Stored *p) {
    uint32_t y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = F::pattern(x[i]);
    if constexpr (sizeof(typename F::Stored) == 2) {
        stream_store(make_uint4(y[0] | y[1] << 16, y[2] | y[3] << 16, y[4] | y[5] << 16, y[6] | y[7] << 16), p);
    } else {
        stream_store(make_uint4(y[0], y[1], y[2], y[3]), reinterpret_cast<uint16_t *>(p));
        stream_store(make_uint4(y[4], y[5], y[6], y[7]), reinterpret_cast<uint16_t *>(p + 4));
    }
}

__device__ __forceinline__ double teacher_logit(const DistillTeacher &t, size_t at) {
    if (t.type == kLogitF32) return (double)static_cast<const float *>(t.logits)[at];
    const uint16_t h = static_cast<const uint16_t *>(t.logits)[at];
    return t.type == kLogitBf16 ? (double)DistillBf16::value(h) : (double)DistillF16::value(h);
}

template <class T, class Op>
__device__ __forceinline__ T wave_fold(T v, Op op) {
#pragma unroll
    for (int step = 32; step > 0; step /= 2) v = op(v, (T)__shfl_xor(v, step));
    return v;
}

// A row's list, one entry a thread: the token (-1: not open, or no entry), its q, the student's logit.
struct Listed { int id; double q, log_q, student; };
// s_part: kDistillMax / 64 entries.  q is 0 for every thread where the row lists nothing.
template <class F>
__device__ __forceinline__ Listed load_list(const DistillTeacher &t, int b, const typename F::Stored *row, const uint32_t *mask, int vocab,
                                            double inv_tau, double *s_part, int tid) {
    constexpr int kWaves = kDistillMax / 64;
    const int lane = tid & 63, wave = tid >> 6;
    Listed e{-1, 0.0, 0.0, 0.0};
    double logit = -(double)INFINITY;
    if (tid < t.k) {
        const int id = t.ids[(size_t)b * t.k + tid];
        if (id >= 0 && id < vocab && (!mask || ((mask[id >> 5] >> (id & 31)) & 1u))) {
            e.student = (double)F::value(row[id]);
            logit = teacher_logit(t, (size_t)b * t.k + tid);
            if (e.student > -(double)INFINITY && logit != -(double)INFINITY) e.id = id;
        }
    }
    if (e.id < 0) logit = -(double)INFINITY;
    double best = wave_fold(logit, [](double x, double y) { return fmax(x, y); });
    if (wave < kWaves && lane == 0) s_part[wave] = best;
    __syncthreads();
    best = s_part[0];
    for (int w = 1; w < kWaves; ++w) best = fmax(best, s_part[w]);
    __syncthreads();
    const double x = (logit - best) * inv_tau;
    e.q = e.id >= 0 ? exp(x) : 0.0;
    double sum = wave_fold(e.q, [](double a, double c) { return a + c; });
    if (wave < kWaves && lane == 0) s_part[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kWaves; ++w) sum += s_part[w];
    __syncthreads();
    e.log_q = x - log(sum);
    e.q = e.id >= 0 ? e.q / sum : 0.0;
    return e;
}

// One block a row: the row's maximum and sum in a first pass, the loss, and with kGrad the gradient in a second.  kForward false: the
// gradient alone, from the numbers that the forward pass has left in `stats`.
template <class F, bool kForward, bool kGrad>
__global__ __launch_bounds__(kDistillBlock) void distill_row_kernel(const typename F::Stored *logits, const uint32_t *__restrict__ bitmask, int vocab,
                                                                   int64_t row_stride, int n_words, DistillTeacher teacher, float scale, double inv_tau,
                                                                   double tau, const float *__restrict__ row_weight, int64_t weight_stride, float *__restrict__ loss,
                                                                   float2 *__restrict__ stats, typename F::Stored *grad, int64_t grad_stride) {
    __shared__ double s_part[kDistillWaves];
    __shared__ float s_top[kDistillWaves];
    __shared__ int s_id[kDistillMax];
    __shared__ double s_q[kDistillMax];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x, whole = vocab >> 3;
    const typename F::Stored *row = logits + (size_t)b * row_stride;
    const uint32_t *mask_words = bitmask ? bitmask + (size_t)b * n_words : nullptr;
    const uint8_t *mask = reinterpret_cast<const uint8_t *>(mask_words);
    const Listed e = load_list<F>(teacher, b, row, mask_words, vocab, inv_tau, s_part, tid);
    const bool live = __syncthreads_or(e.id >= 0);
    float top = -INFINITY, z = 0.0f;           // the maximum; sum of 2^((logit - top) * scale)
    if (kForward && live) {
        // a first look for the maximum, a second for the sum
        auto each = [&](auto fn) {
            for (int g = tid; g < whole; g += kDistillBlock) {
                const uint32_t mu = mask ? mask[g] : 0xFFu;
                if (mu == 0u) continue;
                float x[8];
                load_eight<F>(row + (size_t)g * 8, x);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if ((mu >> k) & 1u) fn(x[k]);
            }
            const int t = whole * 8 + tid;
            if (t < vocab && (!mask || ((mask[t >> 3] >> (t & 7)) & 1u))) fn(F::value(row[t]));
        };
        each([&](float x) { top = fmaxf(top, x); });
        top = wave_fold(top, [](float x, float y) { return fmaxf(x, y); });
        if (lane == 0) s_top[wave] = top;
        __syncthreads();
        for (int w = 0; w < kDistillWaves; ++w) top = fmaxf(top, s_top[w]);
        each([&](float x) { z += __builtin_amdgcn_exp2f((x - top) * scale); });
        double sum = wave_fold((double)z, [](double x, double y) { return x + y; });
        if (lane == 0) s_part[wave] = sum;
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < kDistillWaves; ++w) sum += s_part[w];
        __syncthreads();
        z = (float)sum;
        const double log_z = log(sum);
        double term = e.q > 0.0 || e.q != e.q ? e.q * (e.log_q - ((e.student - (double)top) * inv_tau - log_z)) : 0.0;
        term = wave_fold(term, [](double x, double y) { return x + y; });
        if (lane == 0) s_part[wave] = term;
        __syncthreads();
        if (tid == 0) {
            term = 0.0;
            for (int w = 0; w < kDistillWaves; ++w) term += s_part[w];
            if (loss) loss[b] = (float)(tau * tau * term);
            if (stats) stats[b] = make_float2(top, z);
        }
    } else if (kForward) {
        if (tid == 0) {
            if (loss) loss[b] = 0.0f;
            if (stats) stats[b] = make_float2(0.0f, 1.0f);
        }
    } else {
        const float2 st = stats[b];
        top = st.x;
        z = st.y;
    }
    if (!kGrad) return;
    const double weight = tau * (row_weight ? (double)row_weight[(size_t)b * weight_stride] : 1.0);
    const float share = live ? (float)(weight / (double)z) : 0.0f;
    auto slope = [&](float x) { return x == -INFINITY || !live ? 0.0f : __builtin_amdgcn_exp2f((x - top) * scale) * share; };
    typename F::Stored *out = grad + (size_t)b * grad_stride;
    for (int g = tid; g < whole; g += kDistillBlock) {
        const uint32_t mu = !live ? 0u : mask ? mask[g] : 0xFFu;
        float x[8] = {};
        if (mu != 0u) load_eight<F>(row + (size_t)g * 8, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (mu >> k) & 1u ? slope(x[k]) : 0.0f;
        store_eight<F>(x, out + (size_t)g * 8);
    }
    const int t = whole * 8 + tid;
    if (t < vocab) out[t] = (typename F::Stored)F::pattern(!mask || ((mask[t >> 3] >> (t & 7)) & 1u) ? slope(F::value(row[t])) : 0.0f);
    if (!live) return;
    // the listed tokens, whole: p - q, which may be small beside both, is rounded once
    if (tid < kDistillMax) { s_id[tid] = e.id; s_q[tid] = e.q; }
    __builtin_amdgcn_s_waitcnt(0);             // the row's stores have arrived before these overwrite some of them
    __syncthreads();
    if (tid < teacher.k && e.id >= 0) {
        double q = 0.0;
        bool first = true;                     // of the entries with this token
        for (int j = 0; j < teacher.k; ++j) {
            if (s_id[j] != e.id) continue;
            q += s_q[j];
            if (j < tid) first = false;
        }
        if (first) {
            const double p = (double)__builtin_amdgcn_exp2f(((float)e.student - top) * scale) / (double)z;
            out[e.id] = (typename F::Stored)F::pattern((float)((p - q) * weight));
        }
    }
}

template <class F>
hipError_t launch(const DistillRows &r, const DistillTeacher &teacher, double tau, bool forward, const float *row_weight, int64_t weight_stride, float *loss,
                  float *stats, void *grad, int64_t grad_stride, hipStream_t stream) {
    const int n_words = (r.vocab + 31) / 32;
    const double inv_tau = 1.0 / tau;
    const float scale = (float)(1.44269504088896340736 * inv_tau);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(r.rows), dim3(kDistillBlock), 0, stream, static_cast<const typename F::Stored *>(r.logits), r.bitmask, r.vocab,
                           r.row_stride, n_words, teacher, scale, inv_tau, tau, row_weight, weight_stride, loss, reinterpret_cast<float2 *>(stats),
                           static_cast<typename F::Stored *>(grad), grad_stride);
    };
    if (!forward) go(distill_row_kernel<F, false, true>);
    else if (grad) go(distill_row_kernel<F, true, true>);
    else go(distill_row_kernel<F, true, false>);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_distill(const DistillRows &rows, const DistillTeacher &teacher, double tau, bool forward, const float *row_weight, int64_t weight_stride, float *loss,
                          float *stats, void *grad, int64_t grad_stride, hipStream_t stream) {
    if (rows.rows == 0 || rows.vocab == 0) return hipSuccess;
    switch (rows.type) {
        case kLogitBf16: return launch<DistillBf16>(rows, teacher, tau, forward, row_weight, weight_stride, loss, stats, grad, grad_stride, stream);
        case kLogitF16: return launch<DistillF16>(rows, teacher, tau, forward, row_weight, weight_stride, loss, stats, grad, grad_stride, stream);
        default: return launch<DistillF32>(rows, teacher, tau, forward, row_weight, weight_stride, loss, stats, grad, grad_stride, stream);
    }
}

}  // namespace pre3
