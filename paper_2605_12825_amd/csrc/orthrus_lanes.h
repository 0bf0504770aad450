// Sums, maxima and running sums over the 64 lanes of a wave (device code of the filter and table kernels).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

namespace orthrus {

typedef unsigned long long u64;

// Within a row of sixteen lanes values move without a trip through LDS.

constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;  // DPP: lanes xor 1, xor 2, 7 - i, 15 - i
template <int CTRL> __device__ __forceinline__ float swap_f32(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ u64 swap_u64(u64 x)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, 0xf, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, 0xf, 0xf, true);
    return (u64)hi << 32 | lo;
}
template <int CTRL> __device__ __forceinline__ double swap_f64(double x)
{
    return __longlong_as_double((long long)swap_u64<CTRL>((u64)__double_as_longlong(x)));
}
__device__ __forceinline__ float wave_max(float x)
{
    x = fmaxf(x, swap_f32<kSwap1>(x));
    x = fmaxf(x, swap_f32<kSwap2>(x));
    x = fmaxf(x, swap_f32<kMirror8>(x));
    x = fmaxf(x, swap_f32<kMirror16>(x));
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ double wave_sum(double x)   // the same order in every lane up to mirroring
{
    x += swap_f64<kSwap1>(x);
    x += swap_f64<kSwap2>(x);
    x += swap_f64<kMirror8>(x);
    x += swap_f64<kMirror16>(x);
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
__device__ __forceinline__ u64 wave_sum(u64 x)
{
    x += swap_u64<kSwap1>(x);
    x += swap_u64<kSwap2>(x);
    x += swap_u64<kMirror8>(x);
    x += swap_u64<kMirror16>(x);
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
// A value that all lanes hold, in scalar registers.
__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }
__device__ __forceinline__ double uniform(double x)
{
    return __hiloint2double(__builtin_amdgcn_readfirstlane(__double2hiint(x)), __builtin_amdgcn_readfirstlane(__double2loint(x)));
}
__device__ __forceinline__ u64 lane_value(u64 x, int lane)   // of one lane, for all
{
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}
// Inclusive sum in lane order: shifts within rows of sixteen, then the last lane of a row to the rows behind it.
__device__ __forceinline__ u64 wave_scan(u64 x)
{
    auto step = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, ctrl.value, rows.value, 0xf, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), ctrl.value, rows.value, 0xf, false);
        x += (u64)hi << 32 | lo;
    };
    step(std::integral_constant<int, 0x111>(), std::integral_constant<int, 0xf>());   // row_shr 1, 2, 4, 8
    step(std::integral_constant<int, 0x112>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x114>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x118>(), std::integral_constant<int, 0xf>());
    step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());   // row_bcast 15 to rows 1 and 3
    step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());   // row_bcast 31 to rows 2 and 3
    return x;
}

}  // namespace orthrus
