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

// `wide`: the 16-bit matrix unit, exact.  fp32 and 8-bit outputs (whose scales are
// fp32) always, 16-bit outputs where the caller asks for it: they are then stored
// as fp32 ones are, four of a token by a lane.  bf16 out in the 8-bit unit and exact:
// 16384 slots by 4096 x 3328 205 and 336 us, 65536 of 64 experts by 1024 x 1024 96 and
// 150, 2048 by 1000 x 1512 11.1 and 12.8; of the last, 0.5 % of the outputs differ, in their last bit.
KernelPlan tile_kernel(bool gate, bool fp8, bool wide, TileSize size)
{
    if (fp8) return gate ? plan_of<true, true, true>(size) : plan_of<true, false, true>(size);
    if (wide) return gate ? plan_of<true, true, false>(size) : plan_of<true, false, false>(size);
    return gate ? plan_of<false, true, false>(size) : plan_of<false, false, false>(size);
}

} // namespace eb_product
