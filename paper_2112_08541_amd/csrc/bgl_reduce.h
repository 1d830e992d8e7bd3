// Sums and maxima over neighbouring lanes of a wavefront; every lane gets the result, and the order is the same for all of them.
#pragma once

#include "bgl_internal.h"

namespace bgl {

// Another lane's value: lane ^ 1, lane ^ 2, the mirrored lane of 8 (the other four), the mirrored lane of 16 (the other eight).
template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

// LANES neighbours, a power of two up to 64.
template <int LANES, class F>
__device__ __forceinline__ float across(float v, F both)
{
    if constexpr (LANES >= 2) v = both(v, dpp<0xb1>(v));
    if constexpr (LANES >= 4) v = both(v, dpp<0x4e>(v));
    if constexpr (LANES >= 8) v = both(v, dpp<0x141>(v));
    if constexpr (LANES >= 16) v = both(v, dpp<0x140>(v));
    // Rows of 16, then halves, change places between two registers that hold the same.  (The results go through variables: a bit cast of a
    // vector's element takes its first one, in ROCm 7.2's compiler.)
    if constexpr (LANES >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        const uint32_t a = s[0], b = s[1];
        v = both(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
    }
    if constexpr (LANES >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        const uint32_t a = s[0], b = s[1];
        v = both(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float sum_across(float v)
{
    return across<LANES>(v, [](float a, float b) { return a + b; });
}
template <int LANES>
__device__ __forceinline__ float max_across(float v)
{
    return across<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace bgl
