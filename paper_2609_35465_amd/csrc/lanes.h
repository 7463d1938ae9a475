// Sums and maxima over the lanes of a wave by DPP moves, which take a few cycles
// each where a shuffle goes through LDS.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace tetra_dev {

// v of the lane that the DPP control names, 0 where there is none or the row of
// lanes is masked
template <int CTRL, int ROWS, class T>
__device__ __forceinline__ T dpp(T v) {
    if constexpr (std::is_same_v<T, float>) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, false));
    } else if constexpr (sizeof(T) == 8) {
        const uint64_t u = v;
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), CTRL, ROWS, 0xF, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), CTRL, ROWS, 0xF, false);
        return static_cast<T>(static_cast<uint64_t>(hi) << 32 | lo);
    } else {
        return static_cast<T>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xF, false));
    }
}

template <class T>
__device__ __forceinline__ T lane_of(T v, int lane) {
    if constexpr (std::is_same_v<T, float>) {
        return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    } else if constexpr (sizeof(T) == 8) {
        const uint64_t u = v;
        const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(u), lane);
        const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(u >> 32), lane);
        return static_cast<T>(static_cast<uint64_t>(hi) << 32 | lo);
    } else {
        return static_cast<T>(__builtin_amdgcn_readlane(static_cast<int>(v), lane));
    }
}

// over the lanes up to and with this one: the sum, or of numbers that are not
// negative the maximum
struct Sum {
    template <class T>
    __device__ T operator()(T a, T b) const { return a + b; }
};
struct Max {
    template <class T>
    __device__ T operator()(T a, T b) const { return a > b ? a : b; }
};

template <class F, class T>
__device__ __forceinline__ T row_upto(F f, T v) {      // rows of 16 lanes
    v = f(v, dpp<0x111, 0xF>(v));
    v = f(v, dpp<0x112, 0xF>(v));
    v = f(v, dpp<0x114, 0xF>(v));
    return f(v, dpp<0x118, 0xF>(v));
}

template <class F, class T>
__device__ __forceinline__ T wave_upto(F f, T v) {
    v = row_upto(f, v);
    v = f(v, dpp<0x142, 0xA>(v));
    return f(v, dpp<0x143, 0xC>(v));
}

template <class F, class T>
__device__ __forceinline__ T wave_all(F f, T v) { return lane_of(wave_upto(f, v), 63); }

// f over each LANES (at most 16) neighbouring lanes, in all of them
template <int LANES, class F, class T>
__device__ __forceinline__ T team_all(F f, T v) {
    if constexpr (LANES > 1) v = f(v, dpp<0xB1, 0xF>(v));      // lane ^ 1
    if constexpr (LANES > 2) v = f(v, dpp<0x4E, 0xF>(v));      // lane ^ 2
    if constexpr (LANES > 4) v = f(v, dpp<0x141, 0xF>(v));     // the other four of eight
    if constexpr (LANES > 8) v = f(v, dpp<0x140, 0xF>(v));     // the other eight of sixteen
    return v;
}

// f of the lane's v and that of lane ^ 32, or of lane ^ 16
template <class F>
__device__ __forceinline__ float with_half(F f, float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return f(__builtin_bit_cast(float, static_cast<uint32_t>(r[0])), __builtin_bit_cast(float, static_cast<uint32_t>(r[1])));
}
template <class F>
__device__ __forceinline__ float with_row(F f, float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return f(__builtin_bit_cast(float, static_cast<uint32_t>(r[0])), __builtin_bit_cast(float, static_cast<uint32_t>(r[1])));
}

}  // namespace tetra_dev
