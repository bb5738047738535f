// Sums, maxima and the like over the lanes of a wave, without LDS.
#pragma once
#include "common.h"

namespace vgg {

// Rotations within 16 lanes, then quarters and halves that change places.
template <int N> __device__ __forceinline__ float row_ror(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xf, 0xf, true));
}
template <typename F> __device__ __forceinline__ float quarters(float v, F f)
{
    const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const unsigned q0 = q[0], q1 = q[1];
    return f(__uint_as_float(q0), __uint_as_float(q1));
}
template <typename F> __device__ __forceinline__ float halves(float v, F f)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const unsigned h0 = h[0], h1 = h[1];
    return f(__uint_as_float(h0), __uint_as_float(h1));
}
template <typename F> __device__ __forceinline__ float wave_all(float v, F f)
{
    v = f(v, row_ror<8>(v));
    v = f(v, row_ror<4>(v));
    v = f(v, row_ror<2>(v));
    v = f(v, row_ror<1>(v));
    return halves(quarters(v, f), f);
}
__device__ __forceinline__ float all_max(float v) { return wave_all(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float all_min(float v) { return wave_all(v, [](float a, float b) { return fminf(a, b); }); }
__device__ __forceinline__ float all_sum(float v) { return wave_all(v, [](float a, float b) { return a + b; }); }
// Sums over L neighbouring lanes, L = 8, 16, 32 or 64, in each of them.
template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int L> __device__ __forceinline__ float team_sum(float v)
{
    if constexpr (L == 8) {
        v += dpp<0xB1>(v);      // the other of two lanes,
        v += dpp<0x4E>(v);      // the other two of four,
        return v + dpp<0x141>(v);   // and the other four of eight, mirrored
    } else {
        v += row_ror<8>(v);
        v += row_ror<4>(v);
        v += row_ror<2>(v);
        v += row_ror<1>(v);
        auto add = [](float a, float b) { return a + b; };
        if constexpr (L >= 32) v = quarters(v, add);
        if constexpr (L >= 64) v = halves(v, add);
        return v;
    }
}

}  // namespace vgg
