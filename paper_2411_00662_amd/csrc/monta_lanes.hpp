// Sums and maxima over the lanes of a wave by moves in registers.
#pragma once

#include "monta_device.hpp"

namespace monta {

// op over the L lanes (a power of two, neighbours) that share a number; every one of them gets it.  Steps of 1 and 2 by a permutation of
// four lanes, 4 and 8 by mirrors of 8 and 16 (lanes on one side of a mirror hold the same number by then), 16 and 32 by exchanging rows of
// 16 and halves.  Each step joins the same two groups as a move across the step's distance would.  No LDS: a step through it waits for about 60
// clocks, one here for a few.
template <int L, typename Op>
__device__ __forceinline__ float group_join(float v, [[maybe_unused]] Op op)
{
#if defined(__HIP_DEVICE_COMPILE__)
    auto moved = [](float u, auto ctrl) {
        const int b = __float_as_int(u);
        return __int_as_float(__builtin_amdgcn_update_dpp(b, b, decltype(ctrl)::value, 0xf, 0xf, true));
    };
    if constexpr (L > 1) v = op(v, moved(v, std::integral_constant<int, 0xb1>{}));         // lanes 1 0 3 2
    if constexpr (L > 2) v = op(v, moved(v, std::integral_constant<int, 0x4e>{}));         // lanes 2 3 0 1
    if constexpr (L > 4) v = op(v, moved(v, std::integral_constant<int, 0x141>{}));        // mirror of 8
    if constexpr (L > 8) v = op(v, moved(v, std::integral_constant<int, 0x140>{}));        // mirror of 16
    if constexpr (L > 16) {
        const auto two = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(two[0]), __uint_as_float(two[1]));
    }
    if constexpr (L > 32) {
        const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(two[0]), __uint_as_float(two[1]));
    }
#endif
    return v;
}

template <int L>
__device__ __forceinline__ float group_sum(float v)
{
    return group_join<L>(v, [](float a, float b) { return a + b; });
}

// The larger of two numbers, or the one that is no NaN; no signalling ones.  The instruction itself: around fmaxf the compiler puts others, which make those quiet.
__device__ __forceinline__ float plain_max(float a, float b)
{
#if defined(__HIP_DEVICE_COMPILE__)
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
#else
    return a > b ? a : b;
#endif
}

template <int L>
__device__ __forceinline__ float group_max(float v)
{
    return group_join<L>(v, [](float a, float b) { return plain_max(a, b); });
}

}  // namespace monta
