// Tiles of a product of two matrices in matrix instructions of 16 x 16 results: C[m, n] = sum over k of A[m, k] B[n, k], where each operand lies in
// rows along k or in columns, rows along m or n.
//
// A block makes one tile of kM x kN after the other.  Of every step of 128 bytes (64 numbers of 16 bits) of k it holds both operands' share in LDS, fetched
// there without a way through registers, kStages - 1 steps ahead; the steps of all its tiles are one stream, so that a tile's last steps and what is
// done with its results run while the next tile's first ones are on their way.  What a matrix instruction takes is read from LDS while the one
// before it runs, over the barrier of a step as well.  What bounds it is the fetch: 10 to 11 TB/s over all units, of which a tile of 256 x 256
// makes 1,130 to 1,300 TFLOP/s in bf16 (the instructions alone run at 1,740, and steps of 64 bytes, four waves, or 32 x 32 results gain nothing).
//
// Which of a tile's rows a matrix instruction takes is chosen so that the results of a lane lie side by side: 4 kMi along m and kNj along n where an
// operand lies in rows, eight along m where A lies in columns; results go to memory in pieces of 16 bytes.  LDS holds rows in the order that they are
// read in, and a row's 16-byte pieces at their number xor some bits of the row's, so that what is read at once lies on different banks (the
// fetch writes LDS in the lanes' order: rows and pieces are exchanged in the addresses that it reads).
//
// Of an operand in columns, 16-bit numbers only, a lane reads four numbers of a row along m or n, and sixteen lanes exchange them: each gets four along
// k.  No transposed copy is written: of 1,400 rows and 32,000 x 2,048 bf16 weights both gradients take 390 us, products of transposed copies took 377,
// and the copies 53, and twice the slopes' bytes.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace pre3 {

namespace {

typedef float Float4 __attribute__((ext_vector_type(4)));
typedef int Int4 __attribute__((ext_vector_type(4)));

typedef short Short4 __attribute__((ext_vector_type(4)));
typedef unsigned short Patterns __attribute__((ext_vector_type(8)));
typedef short SignedPatterns __attribute__((ext_vector_type(8)));

// The elements of a product: 16 bytes of them are a lane's share of a matrix instruction's operand.
struct ProductBf16 {
    typedef Float4 Acc;
    typedef __bf16 Frag __attribute__((ext_vector_type(8)));
    static constexpr unsigned short kMostFinite = 0x7F7F;
    __device__ static Acc multiply(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
struct ProductF16 {
    typedef Float4 Acc;
    typedef _Float16 Frag __attribute__((ext_vector_type(8)));
    static constexpr unsigned short kMostFinite = 0x7BFF;
    __device__ static Acc multiply(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
struct ProductI8 {
    typedef Int4 Acc;
    typedef Int4 Frag;
    __device__ static Acc multiply(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

constexpr int kStepBytes = 128;                // of k, of every row: a step
constexpr int kStepRows = kStepBytes / 2;      // and of an operand in columns, in rows

// An operand as it lies: rows along k, or (in columns) along m or n.
struct Operand {
    const char *at;                            // 16-byte aligned
    int64_t stride;                            // bytes from row to row, a multiple of 16
    int rows;                                  // rows beyond are the last one again
    int row_bytes;                             // a multiple of 16; beyond, rows along k have zeros, and rows along m or n their beginning again
    int plane;                                 // bytes from plane to plane, where a number is the sum of several: at another place of the row, or of
};                                             // another row.

// Which planes' products make a product: of two numbers of one part each the one; of a number of one part (A) and a sum of two (B) both; of two sums
// of three parts the six of more than 2^-24 of the largest.  The smallest come first, all along k: the sums are then rounded at the
// products' full size as often as those of numbers of one part, not six times as often.
__device__ __forceinline__ int plane_of_a(int pairs, int pair) { return pairs == 6 ? (0x001102 >> (4 * pair)) & 0xF : 0; }                    // 2 0 1 1 0 0
__device__ __forceinline__ int plane_of_b(int pairs, int pair) { return pairs == 6 ? (0x010120 >> (4 * pair)) & 0xF : pairs - 1 - pair; }     // 0 2 1 0 1 0
constexpr int pairs_of(int planes_a, int planes_b) { return planes_a == 3 ? 6 : planes_b; }

// The next tile of a block: m0 and n0 on, the steps first .. last of k.
struct TileAt { int m, n, m0, n0, first, last; };

template <class T, int kM_, int kN_, int kWavesM_, int kWavesN_, int kStages_, bool kColumnsA_ = false, bool kColumnsB_ = false>
struct ProductTile {
    static constexpr int kM = kM_, kN = kN_, kWavesM = kWavesM_, kWavesN = kWavesN_, kStages = kStages_;
    static constexpr bool kColumnsA = kColumnsA_, kColumnsB = kColumnsB_;
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
    // Of acc[i][j][e] in this lane, within the tile: m_of(i) + e and n_of(j).
    static constexpr int kLaneM = 4 * kMi;
    __device__ static int column_a(int c, int i) { return i / 2 * 32 + c * 8 + ((i ^ c) & 1) * 4; }
    __device__ static int m_of(int i) { return wave() / kWavesN * kMi * 16 + (kColumnsA ? column_a(lane() / 16, i) : lane() / 16 * kLaneM + 4 * i); }
    __device__ static int n_of(int j) { return wave() % kWavesN * kNj * 16 + (kColumnsB ? j * 16 + lane() % 16 : lane() % 16 * kNj + j); }
    // A in columns: eight numbers side by side, of m_of() from the smaller one on, and that one.
    __device__ int eight_of_lane(int i, int j, float x[8]) const {
        const bool odd = lane() / 16 & 1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = odd ? acc[i + 1][j][e] : acc[i][j][e];
            x[e + 4] = odd ? acc[i][j][e] : acc[i + 1][j][e];
        }
        return wave() / kWavesN * kMi * 16 + column_a(lane() / 16, i) / 8 * 8;
    }
    // An operand in rows: the tile's row that is the q-th in LDS, and the piece of it that lies where the first would.
    __device__ static int row_a(int q) { return q / (kMi * 16) * (kMi * 16) + (q % 16 >> 2) * kLaneM + q / 16 % kMi * 4 + (q & 3); }
    __device__ static int row_b(int q) { return q / (kNj * 16) * (kNj * 16) + q % 16 * kNj + q / 16 % kNj; }
    __device__ static int key(int q) { return q & 7; }
    // In columns: the piece of the step's q-th row that lies where the first would.  Half a wave reads eight rows, those of its two sixteens eight apart,
    // and 8 bytes a lane: of B two pieces of each row, of A one half of four pieces.  The rows' numbers go to the other bits of a piece's number among the
    // 16 that a row of all banks has (and to its lowest one: the halves tell A's pieces of a parity apart), so that no two lanes meet.
    template <int kSide, bool kIsA>
    __device__ static int column_key(int q) {
        const int two = q & 3, eight = q >> 3 & 1;
        return (kIsA ? (two & 1) | (two & 2) << 1 | eight << 3 : two << 1 | eight << 3) & (kSide / 8 - 1);
    }
    // One piece of 16 bytes a lane from memory to LDS, the wave's 1,024 bytes in the lanes' order.  A buffer of 4 GiB from the tile's first row on: what
    // is read is held within the operand by its offsets, but for kNowhere, which is beyond the buffer and gives zeros.  (The compiler does not always see
    // that base, `from` and `lds` are one in all lanes.)
    static constexpr uint32_t kNowhere = 0xFFFFFFF0u;
    __device__ static void fetch(uint64_t base, uint32_t offset, uint32_t from, uint32_t lds) {
        constexpr int kRaw32Bit = 0x00020000;
        const Int4 buffer = {__builtin_amdgcn_readfirstlane((int)(uint32_t)base), __builtin_amdgcn_readfirstlane((int)((uint32_t)(base >> 32) & 0xFFFFu)), (int)kNowhere, kRaw32Bit};
        from = __builtin_amdgcn_readfirstlane(from);
        lds = __builtin_amdgcn_readfirstlane(lds);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(buffer), "s"(from) : "memory", "m0");
    }
    template <int kLeft>
    __device__ static void wait_for() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLeft) : "memory"); }
    __device__ static void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

    // One operand's share of the steps, on its way to LDS.
    template <int kSide, int kLoads, bool kColumns, bool kIsA>
    struct Fetches {
        const Operand &of;
        uint64_t base;
        uint32_t offset[kLoads];
        int piece;                                      // of a step (rows): the same in a thread's other rows, which are multiples of 8 on
        __device__ explicit Fetches(const Operand &o) : of(o), base(0), piece(0) {
            const int t = threadIdx.x;
            if constexpr (!kColumns) piece = ((t % 8) ^ key(t / 8)) * 16;
            static_assert(kThreads / 8 % 8 == 0, "rows of a thread");
        }
        __device__ static int column_row(int j) { return (j * kThreads + (int)threadIdx.x) / (kSide / 8); }
        // A tile's first row or column.
        __device__ void enter(int at) {
            const int t = threadIdx.x;
            if constexpr (kColumns) {
                base = (uint64_t)of.at;
#pragma unroll
                for (int j = 0; j < kLoads; ++j) {
                    const int q = column_row(j), column = at * 2 + (((j * kThreads + t) % (kSide / 8)) ^ column_key<kSide, kIsA>(q)) * 16;
                    offset[j] = (uint32_t)(column < of.row_bytes ? column : 0) + (uint32_t)q * (uint32_t)of.stride;
                }
            } else {
                base = (uint64_t)(of.at + (int64_t)at * of.stride);
#pragma unroll
                for (int j = 0; j < kLoads; ++j) {
                    const int q = (j * kThreads + t) / 8;
                    offset[j] = (uint32_t)min(kIsA ? row_a(q) : row_b(q), of.rows - 1 - at) * (uint32_t)of.stride;
                }
            }
        }
        // The step that begins so many bytes along k.
        __device__ void issue(int k, int plane, uint32_t lds) {
            if constexpr (kColumns) {
                const int row = k / 2, most = of.rows - 1 - row;
                const uint64_t from = base + (uint64_t)row * (uint64_t)of.stride;
                const uint32_t at_plane = plane * of.plane;
                if (most >= kStepRows - 1) {
#pragma unroll
                    for (int j = 0; j < kLoads; ++j) fetch(from, offset[j], at_plane, lds + j * kThreads * 16);
                } else {
#pragma unroll
                    for (int j = 0; j < kLoads; ++j) fetch(from, offset[j] - (uint32_t)max(column_row(j) - most, 0) * (uint32_t)of.stride, at_plane, lds + j * kThreads * 16);
                }
            } else {
                const uint32_t along = k + piece, at_plane = plane * of.plane;
                if (k + kStepBytes <= of.row_bytes) {
#pragma unroll
                    for (int j = 0; j < kLoads; ++j) fetch(base, offset[j] + along, at_plane, lds + j * kThreads * 16);
                } else {
#pragma unroll
                    for (int j = 0; j < kLoads; ++j) fetch(base, (int)along < of.row_bytes ? offset[j] + along : kNowhere, at_plane, lds + j * kThreads * 16);
                }
            }
        }
    };

    // A lane's share of a matrix instruction: eight numbers along k, of the i-th row (A) or column (B) of the wave's.
    template <int kSide, int kEach, bool kColumns, bool kIsA>
    __device__ __forceinline__ static typename T::Frag read(const char *lds, uint32_t lds_at, int wave_at, int half, int i) {
        const int l = lane(), r = l & 15;
        if constexpr (kColumns) {
            // lanes 4 e + c of sixteen: row e (and e + 4) of eight along k, and four numbers of it
            const int q = half * 32 + (l >> 4) * 8 + (r >> 2), column = wave_at * kEach * 16 + (kIsA ? column_a(r & 3, i) : i * 16 + (r & 3) * 4);
            auto at = [&](int row) { return lds_at + row * (kSide * 2) + (((column >> 3) ^ column_key<kSide, kIsA>(row)) * 16) + (column & 4) * 2; };
            typedef __attribute__((address_space(3))) Short4 LdsShort4;
            const Short4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(uintptr_t)at(q)), high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(uintptr_t)at(q + 4));
            return __builtin_bit_cast(typename T::Frag, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *reinterpret_cast<const typename T::Frag *>(lds + (wave_at * kEach * 16 + i * 16 + r) * kStepBytes + (((l >> 4) ^ key(r)) * 16 ^ half * 64));
        }
    }
    // What is not finite as the largest number: products with zero stay zero.
    template <bool kWanted>
    __device__ __forceinline__ static typename T::Frag finite(typename T::Frag x) {
        if constexpr (kWanted) {
            // (patterns as signed numbers: those beyond the largest positive one; unsigned: beyond the largest negative one)
            const SignedPatterns above = __builtin_elementwise_min(__builtin_bit_cast(SignedPatterns, x), (SignedPatterns)(short)T::kMostFinite);
            return __builtin_bit_cast(typename T::Frag, __builtin_elementwise_min(__builtin_bit_cast(Patterns, above), (Patterns)(unsigned short)(T::kMostFinite | 0x8000)));
        } else {
            return x;
        }
    }

    // The block's tiles: tiles(i, at) says where the i-th is (false: there is none), done(at) has its sums in acc.
    // The steps of a tile: k_steps for each of so many pairs of planes.  kFiniteA: A's numbers that are not finite count as the largest one.
    template <bool kFiniteA = false, class Tiles, class Done>
    __device__ __forceinline__ void run(const Operand &a, const Operand &b, int pairs, int k_steps, char *lds, Tiles tiles, Done done) {
        const int w = wave();
        const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
        // ---- fetches, ahead of the sums
        TileAt next;
        int next_tile = 0, left = 0, left_of_pair = 0, k = 0, pair = 0, to_stage = 0, on_their_way = 0;
        bool more = true;
        Fetches<kM, kLoadsA, kColumnsA, true> of_a(a);
        Fetches<kN, kLoadsB, kColumnsB, false> of_b(b);
        auto enter = [&]() {                            // the next tile that has steps
            do more = tiles(next_tile++, next);
            while (more && next.first >= next.last);
            if (!more) return;
            const int first = __builtin_amdgcn_readfirstlane(next.first);
            left = __builtin_amdgcn_readfirstlane(next.last) - first;
            // Tiles that wait for memory begin at places of their own along k: rows a power of two apart lie in the same channels, and tiles in
            // step with each other would all ask these (57,344 tokens of 4,096 bf16 numbers, 32 rows: 94 -> 86 us).
            const int from = kN < 256 && !kColumnsA ? __builtin_amdgcn_readfirstlane(next.m0) / kM % k_steps : 0;
            pair = first / k_steps;
            const int at = first - pair * k_steps;
            left_of_pair = k_steps - at;
            k = (from + at < k_steps ? from + at : from + at - k_steps) * kStepBytes;
            of_a.enter(next.m0);
            of_b.enter(next.n0);
        };
        auto issue = [&]() {
            if (!more) return;
            const uint32_t to = lds0 + to_stage * kStageBytes + w * 1024;
            of_a.issue(k, plane_of_a(pairs, pair), to);
            of_b.issue(k, plane_of_b(pairs, pair), to + kM * kStepBytes);
            ++on_their_way;
            to_stage = to_stage + 1 == kStages ? 0 : to_stage + 1;
            k = k + kStepBytes == k_steps * kStepBytes ? 0 : k + kStepBytes;
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
        auto read_x = [&](int half, int i) { x[i] = finite<kFiniteA>(read<kM, kMi, kColumnsA, true>(lds + stage * kStageBytes, lds0 + stage * kStageBytes, w / kWavesN, half, i)); };
        auto read_y = [&](int which, int half, int j) {
            y[which][j] = read<kN, kNj, kColumnsB, false>(lds + stage * kStageBytes + kM * kStepBytes, lds0 + stage * kStageBytes + kM * kStepBytes, w % kWavesN, half, j);
        };
        // multiplies with y[which], and reads the other one and x for what comes next, a half of the present stage
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
            int steps = __builtin_amdgcn_readfirstlane(at.last) - __builtin_amdgcn_readfirstlane(at.first);
            if (steps > 0) {
                advance();
#pragma unroll
                for (int j = 0; j < kNj; ++j) read_y(0, 0, j);
#pragma unroll
                for (int i = 0; i < kMi; ++i) read_x(0, i);
            }
            for (; steps > 0; --steps) {
                multiply(0, 1);
                if (steps > 1) advance();                                // (else what is read is not used)
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

// A launch may have more than 64 KiB of LDS once its kernel is told so, on every device.
inline hipError_t allow_lds(const void *kernel, int bytes) {
    return bytes <= 64 * 1024 ? hipSuccess : hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

}  // namespace

}  // namespace pre3
