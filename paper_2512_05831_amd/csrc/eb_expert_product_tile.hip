// The instantiations of eb_product_tile (eb_expert_product_tile.h).

#include "eb_expert_product_tile.h"

namespace eb_product {

// 16-bit outputs: the 8-bit matrix unit.  fp32 and 8-bit outputs (whose scales
// are fp32): the 16-bit unit, exact.
KernelPlan tile_kernel(bool gate, int32_t out_type)
{
    const bool fp8 = out_type == EB_FP8;
    if (out_type == EB_F16 || out_type == EB_BF16)
        return gate ? tile_plan<TileShape<8, 4, 2, 4, false, true, false>>() : tile_plan<TileShape<8, 4, 2, 4, false, false, false>>();
    if (gate) return fp8 ? tile_plan<TileShape<4, 4, 2, 4, true, true, true>>() : tile_plan<TileShape<4, 4, 2, 4, true, true, false>>();
    return fp8 ? tile_plan<TileShape<4, 4, 2, 4, true, false, true>>() : tile_plan<TileShape<4, 4, 2, 4, true, false, false>>();
}

} // namespace eb_product
