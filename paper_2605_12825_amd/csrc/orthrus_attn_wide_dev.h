// What the translation units of the 64-rows-per-wave attention kernels share next to their body (orthrus_attn_wide.inc).
#pragma once
#include "orthrus_attn_dev.h"

#include <utility>

namespace orthrus {

template <int... S, class F>
__device__ __forceinline__ void for_each_stage(std::integer_sequence<int, S...>, F &&f)
{
    (f(std::integral_constant<int, S>{}), ...);
}

// LDS ring stages: four waves have the CU's LDS to themselves, two workgroups of two waves share it
constexpr int wide_stages(int W) { return W == 4 ? 6 : 4; }

}  // namespace orthrus
