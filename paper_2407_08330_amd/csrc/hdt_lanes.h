// Sums over the lanes of a wave by shifted operands and exchanges, without LDS.
#pragma once

#include <hip/hip_runtime.h>

namespace hdt_lanes {

// (the second operand of an exchange is made opaque: of two results of one value the compiler takes one)
__device__ __forceinline__ unsigned hidden(unsigned x)
{
    asm volatile("" : "+v"(x));
    return x;
}
template <int CTRL>
__device__ __forceinline__ float plus_dpp(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}

// a lane's value and that of the lane 32 further or back, in a fixed order: the lower half-wave's, the upper half-wave's
struct Halves {
    float lower, upper;
};
__device__ __forceinline__ Halves halves(float x)
{
    const unsigned v = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(v, hidden(v), false, false);
    return {__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])};
}
__device__ __forceinline__ float max_halves(float x)
{
    const Halves h = halves(x);
    return fmaxf(h.lower, h.upper);
}
__device__ __forceinline__ float sum_halves(float x)
{
    const Halves h = halves(x);
    return h.lower + h.upper;
}

// the sum over a wave, in every lane
__device__ __forceinline__ float wave_sum(float x)
{
    x = plus_dpp<0xb1>(x);   // lane ^ 1
    x = plus_dpp<0x4e>(x);   // lane ^ 2
    x = plus_dpp<0x141>(x);  // the other quad of eight
    x = plus_dpp<0x140>(x);  // the other eight of a row of 16
    const unsigned v = __builtin_bit_cast(unsigned, x);
    const auto rows = __builtin_amdgcn_permlane16_swap(v, hidden(v), false, false);
    return sum_halves(__builtin_bit_cast(float, (unsigned)rows[0]) + __builtin_bit_cast(float, (unsigned)rows[1]));
}

}  // namespace hdt_lanes
