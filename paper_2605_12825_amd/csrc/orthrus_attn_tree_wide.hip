// Attention of a tree of drafts where arithmetic sets the pace: the 64-rows-per-wave kernel (orthrus_attn_wide.hip) with the tree's
// masks, in a code object of its own.  A wave keeps the paths of its 128 rows' nodes in registers; only the tiles that are masked
// anyway, the ragged one and the block's, look at them.  64 sequences of 1000..2500 tokens, 64 nodes (32/8 heads, 256 rows): 142 us a
// call with 32-row waves -> 134, 0.9 PFLOP/s; bound by issue and the clock under full matrix load, with two items of some 55 tiles to a
// CU their starts and ends are a tenth of it.
#include "orthrus_attn_wide_dev.h"

namespace orthrus {

template <int D, int W, int NS, int MODE, int NT>
__global__ void __launch_bounds__(64 * W, 1) attn_tree_wide_kernel(ATTN_FIRST_PARAMS, const AttnArgs rest)
{
    constexpr bool TREE = true;
#include "orthrus_attn_wide.inc"
}

template <int D, int W>
static auto tree_wide_kernel(const AttnPlan &plan)
{
    if (plan.by_size) return plan.kv_nt ? attn_tree_wide_kernel<D, W, wide_stages(W), kItemsBySize, 1> : attn_tree_wide_kernel<D, W, wide_stages(W), kItemsBySize, 0>;
    return plan.kv_nt ? attn_tree_wide_kernel<D, W, wide_stages(W), kItemsSplit, 1> : attn_tree_wide_kernel<D, W, wide_stages(W), kItemsSplit, 0>;
}

hipError_t launch_tree_wide(const AttnArgs &a, const AttnPlan &plan, int head_dim, dim3 grid, hipStream_t stream)
{
    auto kern = head_dim == 128 ? (plan.waves == 4 ? tree_wide_kernel<128, 4>(plan) : tree_wide_kernel<128, 2>(plan))
                                : (plan.waves == 4 ? tree_wide_kernel<64, 4>(plan) : tree_wide_kernel<64, 2>(plan));
    return launch_timed(kern, grid, dim3(64 * plan.waves), plan.lds_bytes, a, stream, nullptr, 0);
}

}  // namespace orthrus
