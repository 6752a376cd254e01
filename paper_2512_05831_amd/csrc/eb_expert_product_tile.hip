// The instantiations of eb_product_tile (eb_expert_product_tile.h).

#include "eb_expert_product_tile.h"

namespace eb_product {

namespace {

template <bool kWide, bool kFp8>
KernelPlan plan_of(bool gate, bool large)
{
    if (large) return gate ? tile_plan<TileShape<8, 4, 2, 4, kWide, true, kFp8>>() : tile_plan<TileShape<8, 4, 2, 4, kWide, false, kFp8>>();
    if (!gate) return tile_plan<TileShape<4, 4, 2, 2, kWide, false, kFp8>>();
    // 8-bit outputs need their 128 columns in the workgroup.
    if constexpr (kFp8) return tile_plan<TileShape<4, 4, 1, 4, kWide, true, kFp8>>();
    else return tile_plan<TileShape<4, 4, 2, 2, kWide, true, kFp8>>();
}

} // namespace

// 16-bit outputs: the 8-bit matrix unit.  fp32 and 8-bit outputs (whose scales
// are fp32): the 16-bit unit, exact.
KernelPlan tile_kernel(bool gate, int32_t out_type, bool large)
{
    if (out_type == EB_F16 || out_type == EB_BF16) return plan_of<false, false>(gate, large);
    return out_type == EB_FP8 ? plan_of<true, true>(gate, large) : plan_of<true, false>(gate, large);
}

} // namespace eb_product
