// Sums and maxima over the lanes of a wave by moves between lanes, and a barrier for LDS alone.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace pre3 {

namespace {

// Inclusive sums over the lanes of a wave (and lane 63's, in every lane), with moves between lanes: rows of 16 lanes first, then
// the rows' last lanes into the rows behind them.
template <int kControl, int kRows>
__device__ __forceinline__ uint32_t lane_move(uint32_t x) {           // zero where there is no such lane, or the row is not one of kRows
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kControl, kRows, 0xF, kRows == 0xF);
}
template <int kControl, int kRows, class T>
__device__ __forceinline__ T lane_move_of(T x) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, lane_move<kControl, kRows>(__builtin_bit_cast(uint32_t, x)));
    } else {
        const unsigned long long v = __builtin_bit_cast(unsigned long long, x);
        const unsigned long long lo = lane_move<kControl, kRows>((uint32_t)v), hi = lane_move<kControl, kRows>((uint32_t)(v >> 32));
        return __builtin_bit_cast(T, hi << 32 | lo);
    }
}
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
    v += lane_move_of<0x111, 0xF>(v);
    v += lane_move_of<0x112, 0xF>(v);
    v += lane_move_of<0x114, 0xF>(v);
    v += lane_move_of<0x118, 0xF>(v);
    v += lane_move_of<0x142, 0xA>(v);
    v += lane_move_of<0x143, 0xC>(v);
    return v;
}
template <class T>
__device__ __forceinline__ T from_lane(T v, int lane) {         // lane: the same in every lane
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else {
        const unsigned long long x = __builtin_bit_cast(unsigned long long, v);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane);
        return __builtin_bit_cast(T, (unsigned long long)hi << 32 | lo);
    }
}
template <class T>
__device__ __forceinline__ T wave_sum(T v) { return from_lane(wave_scan(v), 63); }
// The largest of a wave's numbers, in every lane.
__device__ __forceinline__ float wave_max(float v) {
    auto step = [&](auto move) { v = fmaxf(v, move(v)); };
    step([](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), 0x111, 0xF, 0xF, false)); });
    step([](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), 0x112, 0xF, 0xF, false)); });
    step([](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), 0x114, 0xF, 0xF, false)); });
    step([](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), 0x118, 0xF, 0xF, false)); });
    step([](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), 0x142, 0xA, 0xF, false)); });
    step([](float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), 0x143, 0xC, 0xF, false)); });
    return from_lane(v, 63);
}

// A barrier that LDS accesses are ordered by; loads on their way stay so.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

}  // namespace

}  // namespace pre3
