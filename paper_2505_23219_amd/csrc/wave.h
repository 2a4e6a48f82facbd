// Sums, maxima and running sums over a wavefront by exchanges inside the registers (DPP): a shuffle goes through the LDS, 0.06 us a step
// of a chain that has six.
#pragma once
#include "common.h"

namespace ghd {

// x of the lane that the control word names; where there is none, or the row of 16 lanes is not in ROWS, `other`
template <int CTRL, int ROWS = 0xf, class T>
__device__ __forceinline__ T lane_from(T x, T other)
{
    static_assert(sizeof(T) == 4 || sizeof(T) == 8, "one or two registers");
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, other), __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
    } else {
        typedef int pair __attribute__((ext_vector_type(2)));
        const pair a = __builtin_bit_cast(pair, x), b = __builtin_bit_cast(pair, other);
        return __builtin_bit_cast(T, (pair){__builtin_amdgcn_update_dpp(b[0], a[0], CTRL, ROWS, 0xf, false),
                                            __builtin_amdgcn_update_dpp(b[1], a[1], CTRL, ROWS, 0xf, false)});
    }
}

// a lane's x in all lanes (lane: uniform)
template <class T>
__device__ __forceinline__ T lane_of(T x, int lane)
{
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
    } else {
        typedef int pair __attribute__((ext_vector_type(2)));
        const pair a = __builtin_bit_cast(pair, x);
        return __builtin_bit_cast(T, (pair){__builtin_amdgcn_readlane(a[0], lane), __builtin_amdgcn_readlane(a[1], lane)});
    }
}

// op over the lanes up to and with this one; none: op(none, x) is x
template <class T, class Op>
__device__ __forceinline__ T wave_running(T x, T none, Op op)
{
    x = op(lane_from<0x111>(x, none), x);              // row_shr: 1, 2, 4, 8 lanes up inside a row
    x = op(lane_from<0x112>(x, none), x);
    x = op(lane_from<0x114>(x, none), x);
    x = op(lane_from<0x118>(x, none), x);
    x = op(lane_from<0x142, 0xa>(x, none), x);         // row_bcast15: a row's last lane to the next row
    return op(lane_from<0x143, 0xc>(x, none), x);      // row_bcast31: lane 31 to the second half
}
template <class T>
__device__ __forceinline__ T running_sum(T x)
{
    return wave_running(x, (T)0, [](T a, T b) { return a + b; });
}
// in all lanes
template <class T>
__device__ __forceinline__ T wave_sum(T x)
{
    return lane_of(running_sum(x), 63);
}
__device__ __forceinline__ float wave_highest(float x)
{
    return lane_of(wave_running(x, -INFINITY, [](float a, float b) { return fmaxf(a, b); }), 63);
}
__device__ __forceinline__ int wave_highest(int x)
{
    return lane_of(wave_running(x, (int)0x80000000, [](int a, int b) { return max(a, b); }), 63);
}
__device__ __forceinline__ uint32_t wave_highest(uint32_t x)
{
    return lane_of(wave_running(x, 0u, [](uint32_t a, uint32_t b) { return max(a, b); }), 63);
}

}  // namespace ghd
