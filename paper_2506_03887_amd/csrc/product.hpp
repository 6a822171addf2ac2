// Tiles of a product of two matrices that both lie with the summed dimension contiguous: C[m, n] = sum over k of A[m, k] B[n, k], in
// matrix instructions of 16 x 16 results.
//
// A block makes kM x kN of them.  Of every step of 128 bytes of k it holds the rows of both operands in LDS, fetched there without a way
// through registers, kStages - 1 steps ahead.  A row's eight 16-byte pieces lie at their number xor the row's lowest three bits, so that the
// sixteen rows that a wave reads at one k are on different banks (the fetch writes LDS in the lanes' order: the pieces are exchanged in the
// addresses that it reads).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace pre3 {

namespace {

typedef float Float4 __attribute__((ext_vector_type(4)));
typedef int Int4 __attribute__((ext_vector_type(4)));

// The elements of a product: 16 bytes of them are a lane's share of a matrix instruction's operand.
struct ProductBf16 {
    typedef Float4 Acc;
    typedef __bf16 Frag __attribute__((ext_vector_type(8)));
    static constexpr int kBytes = 2;
    __device__ static Acc multiply(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
struct ProductF16 {
    typedef Float4 Acc;
    typedef _Float16 Frag __attribute__((ext_vector_type(8)));
    static constexpr int kBytes = 2;
    __device__ static Acc multiply(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
struct ProductI8 {
    typedef Int4 Acc;
    typedef Int4 Frag;
    static constexpr int kBytes = 1;
    __device__ static Acc multiply(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

constexpr int kStepBytes = 128;                // of k that a step takes of every row

// Rows of an operand.  A row holds one plane of `row_bytes` of k, or three side by side (a 32-bit number as the sum of three of 16 bits).
struct Operand {
    const char *at;                            // 16-byte aligned
    int64_t stride;                            // bytes from row to row, a multiple of 16
    int rows;                                  // rows beyond are the last one again
    int row_bytes;                             // of a plane, a multiple of 16.  What a step reads beyond is the row's beginning again,
};                                             // against which the other operand has zeros

// Which planes' products make the product of two sums of three parts: all of more than 2^-24 of the largest.
constexpr int kPlanePairs = 6;
__device__ __forceinline__ int plane_of_a(int pair) { return (0x211000 >> (4 * pair)) & 0xF; }      // 0 0 0 1 1 2
__device__ __forceinline__ int plane_of_b(int pair) { return (0x010210 >> (4 * pair)) & 0xF; }      // 0 1 2 0 1 0

template <class T, int kM_, int kN_, int kWavesM_, int kWavesN_, int kStages_>
struct ProductTile {
    static constexpr int kM = kM_, kN = kN_, kWavesM = kWavesM_, kWavesN = kWavesN_, kStages = kStages_;
    static constexpr int kThreads = kWavesM * kWavesN * 64;
    static constexpr int kMi = kM / kWavesM / 16, kNj = kN / kWavesN / 16;           // 16 x 16 results of a wave
    static constexpr int kLoadsA = kM * 8 / kThreads, kLoadsB = kN * 8 / kThreads;   // 16-byte pieces that a thread fetches of a step
    static constexpr int kStageBytes = (kM + kN) * kStepBytes;
    static constexpr int kLdsBytes = kStages * kStageBytes;
    static_assert(kLoadsA * kThreads == kM * 8 && kLoadsB * kThreads == kN * 8, "whole fetches");
    static_assert(kMi * kWavesM * 16 == kM && kNj * kWavesN * 16 == kN, "whole results");
    static_assert((kStages - 1) * (kLoadsA + kLoadsB) < 64, "the counter of loads on their way");
    static_assert(kLdsBytes <= 160 * 1024, "LDS of a unit");

    typename T::Acc acc[kMi][kNj];

    __device__ static int wave() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }
    __device__ static int lane() { return (int)threadIdx.x & 63; }
    // Of acc[i][j][e] in this lane: m and n within the tile.
    __device__ static int m_of(int i) { return (wave() / kWavesN * kMi + i) * 16 + lane() / 16 * 4; }      // + e
    __device__ static int n_of(int j) { return (wave() % kWavesN * kNj + j) * 16 + lane() % 16; }

    // One piece of 16 bytes a lane from memory to LDS, the wave's 1,024 bytes in the lanes' order.
    __device__ static void fetch(Int4 buffer, uint32_t offset, uint32_t from, uint32_t lds) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(buffer), "s"(from) : "memory", "m0");
    }
    template <int kLeft>
    __device__ static void wait_and_meet() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kLeft) : "memory"); }
    __device__ static Int4 buffer_of(const char *at) {
        const uint64_t p = (uint64_t)at;
        constexpr int kRaw32Bit = 0x00020000;
        // (whole 4 GiB from here: what is read is held within the operand by its offsets)
        return Int4{__builtin_amdgcn_readfirstlane((int)(uint32_t)p), __builtin_amdgcn_readfirstlane((int)((uint32_t)(p >> 32) & 0xFFFFu)), -1, kRaw32Bit};
    }

    // Sums the steps `first` .. `last` of k into acc, of rows m0 and n0 on.  planes: 3 where both operands hold three; a step is then one pair of planes.
    __device__ __forceinline__ void run(const Operand &a, const Operand &b, int m0, int n0, int planes, int first, int last, char *lds) {
        const int t = threadIdx.x, w = wave(), l = lane();
#pragma unroll
        for (int i = 0; i < kMi; ++i)
#pragma unroll
            for (int j = 0; j < kNj; ++j) acc[i][j] = typename T::Acc{0, 0, 0, 0};
        if (first >= last) return;
        const Int4 buffer_a = buffer_of(a.at + (int64_t)m0 * a.stride), buffer_b = buffer_of(b.at + (int64_t)n0 * b.stride);
        const int piece = ((t & 7) ^ ((t >> 3) & 7)) * 16;
        uint32_t row_a[kLoadsA], row_b[kLoadsB];
#pragma unroll
        for (int j = 0; j < kLoadsA; ++j) row_a[j] = (uint32_t)min(j * (kThreads / 8) + (t >> 3), a.rows - 1 - m0) * (uint32_t)a.stride;
#pragma unroll
        for (int j = 0; j < kLoadsB; ++j) row_b[j] = (uint32_t)min(j * (kThreads / 8) + (t >> 3), b.rows - 1 - n0) * (uint32_t)b.stride;
        const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
        auto issue = [&](int step, int stage) {
            int k = step, plane_a = 0, plane_b = 0;
            if (planes > 1) {
                k = step / kPlanePairs;
                const int pair = step - k * kPlanePairs;
                plane_a = plane_of_a(pair) * a.row_bytes;
                plane_b = plane_of_b(pair) * b.row_bytes;
            }
            const int at = k * kStepBytes + piece;
            const uint32_t at_a = (uint32_t)(at < a.row_bytes ? at : 0), at_b = (uint32_t)(at < b.row_bytes ? at : 0);
            const uint32_t to = lds0 + stage * kStageBytes + w * 1024;
#pragma unroll
            for (int j = 0; j < kLoadsA; ++j) fetch(buffer_a, row_a[j] + at_a, plane_a, to + j * kThreads * 16);
#pragma unroll
            for (int j = 0; j < kLoadsB; ++j) fetch(buffer_b, row_b[j] + at_b, plane_b, to + kM * kStepBytes + j * kThreads * 16);
        };
        const int r = l & 15, sw = ((l >> 4) ^ (l & 7)) * 16;               // of the first four pieces; the last four's differ in bit 2
        const int from_a = (w / kWavesN * kMi * 16 + r) * kStepBytes + sw, from_b = kM * kStepBytes + (w % kWavesN * kNj * 16 + r) * kStepBytes + sw;
#pragma unroll
        for (int s = 0; s < kStages - 1; ++s)
            if (first + s < last) issue(first + s, s);
        int stage = 0, ahead = kStages - 1;
        for (int step = first; step < last; ++step) {
            // this step's pieces are there, of all waves, and all have read the step before
            if (step + kStages - 2 < last) wait_and_meet<(kStages - 2) * (kLoadsA + kLoadsB)>();
            else wait_and_meet<0>();
            if (step + kStages - 1 < last) issue(step + kStages - 1, ahead);
            const char *now = lds + stage * kStageBytes;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                typename T::Frag x[kMi], y[kNj];
#pragma unroll
                for (int j = 0; j < kNj; ++j) y[j] = *reinterpret_cast<const typename T::Frag *>(now + ((from_b + j * 16 * kStepBytes) ^ (half * 64)));
#pragma unroll
                for (int i = 0; i < kMi; ++i) x[i] = *reinterpret_cast<const typename T::Frag *>(now + ((from_a + i * 16 * kStepBytes) ^ (half * 64)));
#pragma unroll
                for (int i = 0; i < kMi; ++i)
#pragma unroll
                    for (int j = 0; j < kNj; ++j) acc[i][j] = T::multiply(x[i], y[j], acc[i][j]);
            }
            stage = stage + 1 == kStages ? 0 : stage + 1;
            ahead = ahead + 1 == kStages ? 0 : ahead + 1;
        }
    }
};

// The tile of a block: blocks go to the eight dies in turn, each of which has a cache of its own.  A die's blocks take neighbouring tiles: eight
// along n at one m, then the next m.
constexpr int kDies = 8;
__device__ __forceinline__ void tile_of_block(int block, int tiles_m, int tiles_n, int &m, int &n) {
    const int total = tiles_m * tiles_n, each = total / kDies, more = total % kDies, die = block % kDies;
    int at = die * each + min(die, more) + block / kDies;
    constexpr int kAlong = 8;
    const int band = at / (tiles_m * kAlong), width = min(kAlong, tiles_n - band * kAlong);
    at -= band * tiles_m * kAlong;
    m = at / width;
    n = band * kAlong + at % width;
}

}  // namespace

}  // namespace pre3
