// The instantiations of eb_product_tile (eb_expert_product_tile.h).

#include "eb_expert_product_tile.h"

namespace eb_product {

namespace {

template <bool kWide, bool kGate, bool kFp8>
KernelPlan plan_of(TileSize size)
{
    if (size == TileSize::kHuge) return tile_plan<TileShape<8, 4, 2, kWide, kGate, kFp8>>();
    if (size == TileSize::kLarge) return tile_plan<TileShape<8, 4, 1, kWide, kGate, kFp8>>();
    // Gated 8-bit outputs: 256 rows too, for a whole block of outputs.
    constexpr int kRows = kGate && kFp8 ? 4 : 2;
    if (size == TileSize::kMedium) return tile_plan<TileShape<4, kRows, 1, kWide, kGate, kFp8>>();
    return tile_plan<TileShape<2, kRows, 1, kWide, kGate, kFp8>>();
}

} // namespace

// 16-bit outputs: the 8-bit matrix unit.  fp32 and 8-bit outputs (whose scales
// are fp32): the 16-bit unit, exact.
KernelPlan tile_kernel(bool gate, int32_t out_type, TileSize size)
{
    if (out_type == EB_F16 || out_type == EB_BF16) return gate ? plan_of<false, true, false>(size) : plan_of<false, false, false>(size);
    if (out_type == EB_FP8) return gate ? plan_of<true, true, true>(size) : plan_of<true, false, true>(size);
    return gate ? plan_of<true, true, false>(size) : plan_of<true, false, false>(size);
}

} // namespace eb_product
