// Sums and largest values over groups of neighbouring lanes, in every lane of the group, without LDS.
#pragma once
#include <hip/hip_runtime.h>

namespace {

template <int CONTROL>
__device__ __forceinline__ float moved(float v)
{
    return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CONTROL, 0xf, 0xf, true));
}

// LANES a power of two up to 64.  All lanes of a group get the same bits: every step adds the same two numbers in both lanes.
template <int LANES>
__device__ __forceinline__ float group_sum(float v)
{
    if constexpr (LANES >= 2) v += moved<0xB1>(v);          // lane ^ 1
    if constexpr (LANES >= 4) v += moved<0x4E>(v);          // lane ^ 2
    if constexpr (LANES >= 8) v += moved<0x141>(v);         // mirrored within eight: the other four's sum
    if constexpr (LANES >= 16) v += moved<0x140>(v);        // mirrored within sixteen
    if constexpr (LANES >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if constexpr (LANES >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}

// The largest value of a wavefront.
__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, moved<0xB1>(v));
    v = fmaxf(v, moved<0x4E>(v));
    v = fmaxf(v, moved<0x141>(v));
    v = fmaxf(v, moved<0x140>(v));
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
    const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(t[0]), __uint_as_float(t[1]));
}

}  // namespace
