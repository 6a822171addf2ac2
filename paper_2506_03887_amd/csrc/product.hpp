// Tiles of a product of two matrices that both lie with the summed dimension contiguous: C[m, n] = sum over k of A[m, k] B[n, k], in
// matrix instructions of 16 x 16 results.
//
// A block makes one tile of kM x kN after the other.  Of every step of kStep bytes of k it holds the rows of both operands in LDS, fetched there
// without a way through registers, kStages - 1 steps ahead; the steps of all its tiles are one stream, so that a tile's last steps and what is
// done with its results run while the next tile's first ones are on their way.  What a matrix instruction takes is read from LDS while the one
// before it runs, over the barrier of a step as well.
//
// Which of a tile's rows a matrix instruction takes is chosen so that the results of a lane lie side by side: 4 kMi along m and kNj along n,
// and results go to memory in pieces of 16 bytes, of which a wave's make whole lines.  LDS holds the rows in the order that they are read
// in, and a row's 16-byte pieces at their number xor some bits of the row's, so that eight rows that are read at one k lie on different banks
// (the fetch writes LDS in the lanes' order: rows and pieces are exchanged in the addresses that it reads).
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

constexpr int kStepBytes = 128;                // what k is padded to: the longest step of a row

// Rows of an operand.  A row holds one plane of `row_bytes` of k, or three side by side (a 32-bit number as the sum of three of 16 bits).
struct Operand {
    const char *at;                            // 16-byte aligned
    int64_t stride;                            // bytes from row to row, a multiple of 16
    int rows;                                  // rows beyond are the last one again
    int row_bytes;                             // of a plane, a multiple of 16.  What a step reads beyond is the row's beginning again,
};                                             // against which the other operand has zeros

// Which planes' products make a product: of two numbers of one part each the one; of a number of one part (A) and a sum of two (B) both; of two sums
// of three parts the six of more than 2^-24 of the largest.  The smallest come first, all along k: the sums are then rounded at the
// products' full size as often as those of numbers of one part (32-bit operands of 7,680 numbers: a loss is off by 2.2e-6 instead of 4.2e-6).
__device__ __forceinline__ int plane_of_a(int pairs, int pair) { return pairs == 6 ? (0x001102 >> (4 * pair)) & 0xF : 0; }                    // 2 0 1 1 0 0
__device__ __forceinline__ int plane_of_b(int pairs, int pair) { return pairs == 6 ? (0x010120 >> (4 * pair)) & 0xF : pairs - 1 - pair; }     // 0 2 1 0 1 0
constexpr int pairs_of(int planes_a, int planes_b) { return planes_a == 3 ? 6 : planes_b; }

// The next tile of a block: rows m0 and n0 on, the steps first .. last of k (an even number of them where they have 64 bytes).
struct TileAt { int m, n, m0, n0, first, last; };

template <class T, int kM_, int kN_, int kWavesM_, int kWavesN_, int kStep_, int kStages_>
struct ProductTile {
    static constexpr int kM = kM_, kN = kN_, kWavesM = kWavesM_, kWavesN = kWavesN_, kStep = kStep_, kStages = kStages_;
    static constexpr int kThreads = kWavesM * kWavesN * 64;
    static constexpr int kMi = kM / kWavesM / 16, kNj = kN / kWavesN / 16;                      // 16 x 16 results of a wave
    static constexpr int kPieces = kStep / 16, kHalves = kStep / 64;                            // of a row's step; matrix instructions along it
    static constexpr int kLoadsA = kM * kPieces / kThreads, kLoadsB = kN * kPieces / kThreads;  // pieces that a thread fetches of a step
    static constexpr int kStageBytes = (kM + kN) * kStep;
    static constexpr int kLdsBytes = kStages * kStageBytes;
    static_assert(kStep == 64 || kStep == 128, "a step");
    static_assert(kLoadsA * kThreads == kM * kPieces && kLoadsB * kThreads == kN * kPieces, "whole fetches");
    static_assert(kMi * kWavesM * 16 == kM && kNj * kWavesN * 16 == kN, "whole results");
    static_assert((kStages - 1) * (kLoadsA + kLoadsB) < 64, "the counter of loads on their way");
    static_assert(kLdsBytes <= 160 * 1024, "LDS of a unit");

    typename T::Acc acc[kMi][kNj];

    __device__ static int wave() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }
    __device__ static int lane() { return (int)threadIdx.x & 63; }
    // Of acc[i][j][e] in this lane, within the tile: m_of() + 4 i + e and n_of() + j.
    static constexpr int kLaneM = 4 * kMi;
    __device__ static int m_of() { return wave() / kWavesN * kMi * 16 + lane() / 16 * kLaneM; }
    __device__ static int n_of() { return wave() % kWavesN * kNj * 16 + lane() % 16 * kNj; }
    // The row of the tile that is the q-th in LDS, and the piece of it that lies where the first would.
    __device__ static int row_a(int q) { return q / (kMi * 16) * (kMi * 16) + (q % 16 >> 2) * kLaneM + q / 16 % kMi * 4 + (q & 3); }
    __device__ static int row_b(int q) { return q / (kNj * 16) * (kNj * 16) + q % 16 * kNj + q / 16 % kNj; }
    __device__ static int key(int q) { return kStep == 128 ? q & 7 : q >> 1 & 3; }

    // One piece of 16 bytes a lane from memory to LDS, the wave's 1,024 bytes in the lanes' order.  A buffer of 4 GiB from the tile's first row on: what
    // is read is held within the operand by its offsets.  (The compiler does not always see that base, `from` and `lds` are one in all lanes.)
    __device__ static void fetch(uint64_t base, uint32_t offset, uint32_t from, uint32_t lds) {
        constexpr int kRaw32Bit = 0x00020000;
        const Int4 buffer = {__builtin_amdgcn_readfirstlane((int)(uint32_t)base), __builtin_amdgcn_readfirstlane((int)((uint32_t)(base >> 32) & 0xFFFFu)), -1, kRaw32Bit};
        from = __builtin_amdgcn_readfirstlane(from);
        lds = __builtin_amdgcn_readfirstlane(lds);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(buffer), "s"(from) : "memory", "m0");
    }
    template <int kLeft>
    __device__ static void wait_for() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLeft) : "memory"); }
    __device__ static void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

    // The block's tiles: tiles(i, at) says where the i-th is (false: there is none), done(at) has its sums in acc.
    // The steps of a tile: k_steps for each of so many pairs of planes.
    template <class Tiles, class Done>
    __device__ __forceinline__ void run(const Operand &a, const Operand &b, int pairs, int k_steps, char *lds, Tiles tiles, Done done) {
        const int t = threadIdx.x, w = wave(), l = lane();
        const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + w * 1024;
        // ---- fetches, ahead of the sums
        TileAt next;
        int next_tile = 0, left = 0, left_of_pair = 0, from_k = 0, k = 0, pair = 0, to_stage = 0, on_their_way = 0;
        bool more = true;
        uint64_t base_a = 0, base_b = 0;
        uint32_t from_a[kLoadsA], from_b[kLoadsB];
        const int piece = ((t % kPieces) ^ key(t / kPieces)) * 16;       // (the same in a thread's other rows: they are multiples of 8 on)
        static_assert(kThreads / kPieces % 8 == 0, "rows of a thread");
        auto enter = [&]() {                            // the next tile that has steps
            do more = tiles(next_tile++, next);
            while (more && next.first >= next.last);
            if (!more) return;
            const int first = __builtin_amdgcn_readfirstlane(next.first);
            left = __builtin_amdgcn_readfirstlane(next.last) - first;
            // Tiles that wait for memory begin at places of their own along k: rows a power of two apart lie in the same channels, and tiles in
            // step with each other would all ask these (57,344 tokens of 4,096 bf16 numbers, 32 rows: 94 -> 86 us).
            from_k = kN < 256 ? __builtin_amdgcn_readfirstlane(next.m0) / kM % k_steps : 0;
            pair = first / k_steps;
            const int at = first - pair * k_steps;
            left_of_pair = k_steps - at;
            k = (from_k + at < k_steps ? from_k + at : from_k + at - k_steps) * kStep;
            base_a = (uint64_t)(a.at + (int64_t)next.m0 * a.stride);
            base_b = (uint64_t)(b.at + (int64_t)next.n0 * b.stride);
#pragma unroll
            for (int j = 0; j < kLoadsA; ++j) from_a[j] = (uint32_t)min(row_a((j * kThreads + t) / kPieces), a.rows - 1 - next.m0) * (uint32_t)a.stride;
#pragma unroll
            for (int j = 0; j < kLoadsB; ++j) from_b[j] = (uint32_t)min(row_b((j * kThreads + t) / kPieces), b.rows - 1 - next.n0) * (uint32_t)b.stride;
        };
        auto issue = [&]() {
            if (!more) return;
            const int at = k + piece, plane_a = plane_of_a(pairs, pair) * a.row_bytes, plane_b = plane_of_b(pairs, pair) * b.row_bytes;
            const uint32_t at_a = at < a.row_bytes ? at : 0, at_b = at < b.row_bytes ? at : 0, to = lds0 + to_stage * kStageBytes;
#pragma unroll
            for (int j = 0; j < kLoadsA; ++j) fetch(base_a, from_a[j] + at_a, plane_a, to + j * kThreads * 16);
#pragma unroll
            for (int j = 0; j < kLoadsB; ++j) fetch(base_b, from_b[j] + at_b, plane_b, to + kM * kStep + j * kThreads * 16);
            ++on_their_way;
            to_stage = to_stage + 1 == kStages ? 0 : to_stage + 1;
            k = k + kStep == k_steps * kStep ? 0 : k + kStep;
            if (--left_of_pair == 0) { ++pair; left_of_pair = k_steps; }      // (k is back where it began)
            if (--left == 0) enter();
        };
        enter();
#pragma nounroll
        for (int s = 0; s < kStages - 1; ++s) issue();
        // ---- sums
        int stage = -1;
        bool there = false;                             // the next step's pieces, of this wave
        auto wait = [&]() {
            if (there) return;
            if (on_their_way == kStages - 1) wait_for<(kStages - 2) * (kLoadsA + kLoadsB)>();
            else wait_for<0>();
        };
        // The next step's pieces are there, of all waves, and all have read the step before it, whose place the next fetch takes.
        auto advance = [&]() {
            wait();
            there = false;
            meet();
            --on_their_way;
            issue();
            stage = stage + 1 == kStages ? 0 : stage + 1;
        };
        // A step's operands: those along m one at a time, read again as soon as they have been multiplied, those along n twice.
        typename T::Frag x[kMi], y[2][kNj];
        const int r = l & 15, at_a = (w / kWavesN * kMi * 16 + r) * kStep, at_b = kM * kStep + (w % kWavesN * kNj * 16 + r) * kStep, at_piece = ((l >> 4) ^ key(r)) * 16;
        auto read_x = [&](int half, int i) { x[i] = *reinterpret_cast<const typename T::Frag *>(lds + stage * kStageBytes + (at_piece ^ half * 64) + at_a + i * 16 * kStep); };
        auto read_y = [&](int which, int half, int j) { y[which][j] = *reinterpret_cast<const typename T::Frag *>(lds + stage * kStageBytes + (at_piece ^ half * 64) + at_b + j * 16 * kStep); };
        // multiplies with y[which], and reads the other one and x for what comes next, a half of the present stage.
        auto multiply = [&](int which, int half) {
#pragma unroll
            for (int i = 0; i < kMi; ++i) {
#pragma unroll
                for (int j = i * kNj / kMi; j < (i + 1) * kNj / kMi; ++j) read_y(which ^ 1, half, j);
#pragma unroll
                for (int j = 0; j < kNj; ++j) acc[i][j] = T::multiply(x[i], y[which][j], acc[i][j]);
                read_x(half, i);
            }
        };
        TileAt at;
        for (int i_tile = 0; tiles(i_tile, at); ++i_tile) {
#pragma unroll
            for (int i = 0; i < kMi; ++i)
#pragma unroll
                for (int j = 0; j < kNj; ++j) acc[i][j] = typename T::Acc{0, 0, 0, 0};
            // (steps of 64 bytes come in pairs)
            int turns = (__builtin_amdgcn_readfirstlane(at.last) - __builtin_amdgcn_readfirstlane(at.first)) * kHalves / 2;
            if (turns > 0) {
                advance();
#pragma unroll
                for (int j = 0; j < kNj; ++j) read_y(0, 0, j);
#pragma unroll
                for (int i = 0; i < kMi; ++i) read_x(0, i);
            }
            for (; turns > 0; --turns) {
                if constexpr (kHalves == 1) advance();
                multiply(0, kHalves - 1);
                if (turns > 1) advance();                                // (else what is read is not used)
                multiply(1, 0);
            }
            // (waited for now: behind the results' stores the wait would be for these as well)
            if (on_their_way > 0 && !there) { wait(); there = true; }
            done(at);
        }
    }
};

// Where the tile number `at` lies.  Blocks go to the eight dies in turn, each of which has a cache of its own: a die's blocks take neighbouring tiles,
// eight along n at one m, then the next m.  blocks: of the launch, each of which takes every blocks-th tile.
constexpr int kDies = 8, kUnits = 256;
__device__ __forceinline__ void place_of_tile(int at, int tiles_m, int tiles_n, int &m, int &n) {
    const int total = tiles_m * tiles_n, each = total / kDies, more = total % kDies, die = at % kDies;
    at = die * each + min(die, more) + at / kDies;
    constexpr int kAlong = 8;
    const int band = at / (tiles_m * kAlong), width = min(kAlong, tiles_n - band * kAlong);
    at -= band * tiles_m * kAlong;
    m = at / width;
    n = band * kAlong + at % width;
}

}  // namespace

}  // namespace pre3
