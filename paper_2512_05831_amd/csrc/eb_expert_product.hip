// eb_expert_product (include/eb_experts.h): checks of arguments and the choice
// of its kernel.

#include <hip/hip_runtime.h>

#include <stdint.h>

#include <algorithm>
#include <limits>

#include "eb_expert_product.h"
#include "eb_internal.h"

namespace {

using namespace eb_product;
using eb_detail::fail;

constexpr int64_t kMostSize = (int64_t)1 << 30;

int element_bytes(int32_t type) { return type == EB_F32 ? 4 : type == EB_FP8 ? 1 : 2; }

// The kernel for a call, from its mean of slots per expert (the counts are on
// the device) and how many pieces of so many slots by so many weight rows it then
// has.  Measured, us of GPU time a call, with slots a third around the mean:
//   Stream against small tiles.  Its time is its pieces', 16 by 16, whatever the
//   other's is per block of K.  8-bit unit: one expert of 1000 x 1520, 200 slots (819
//   pieces) 6.5 and 7.7, 300 slots (1197) 7.9 and 7.7; of 2048 x 4096, 64 slots (512) 10.7
//   and 19.7, 200 slots (1664) 25.2 and 20.1; 4 experts of 1024 x 512, 64 slots (1024) 6.9
//   and 5.3; a gate changes little.  16-bit unit: 1000 x 1520, 200 slots 7.7 and 9.4; 2048 x
//   4096, 128 slots (1024) 18.7 and 20.6, 200 slots 28.5 and 20.7; 16 experts of 1024 x
//   1024, 8 slots (1024) 6.9 and 7.3.  For 8-bit outputs a workgroup holds 128 rows (with a
//   gate 256): 1000 x 1520 9.2 and 9.8, but 2048 x 4096 25.3 and 20.6, 1024 x 512 7.1 and 6.2.
//   Larger tiles read their operands less often, smaller ones fill the GPU and
//   waste less of an expert's last tile.  Huge against large, 16384 slots of one
//   expert of 4096 x 3328: 195 and 213 in the 8-bit unit, 346 and 363 in the 16-bit
//   one; 64 experts of 2048 x 3328, 512 slots each: 287 and 272, gated with 8-bit
//   outputs 470 and 417; 2048 slots each: equal within 1 %.  16 experts of 2048 x
//   1024: large against medium (of 256 rows), 8-bit unit, 200 slots (256 tiles) 16.8
//   and 17.8, 900 slots 43.6 and 46.2; 16-bit unit 200 slots 33.8 and 25.0, 400 slots
//   (512 tiles) 41.6 and 44.0.
//   Medium against small, 16-bit unit: 4000 slots by 1000 x 1520 (504 tiles) 18.0 and
//   20.5, 16 experts of 512 x 2048 with 375 slots (384) 22.1 and 24.2; but 32 experts
//   of 1024 x 2048 with 100 slots (512) 29.9 and 26.6.  8-bit unit: 16 experts of 512 x
//   2048 with 375 slots 15.4 and 18.7 (medium of 256 rows).  Pieces are counted with 128
//   rows where medium and small tiles have 256 too (a gate with 8-bit outputs).  Tiles against
//   each other have not been timed for means below 100 slots, nor for one GPU's shard, whose
//   M holds every GPU's slots.
KernelPlan choose_kernel(int64_t M, int32_t E, int64_t N, int64_t ldx, int64_t ldw, bool gathered, int64_t x_rows, bool gate,
                         int32_t out_type, bool exact)
{
    const bool fp8 = out_type == EB_FP8, wide = fp8 || out_type == EB_F32 || exact;
    // The tile kernel addresses x (a slot tile's rows, or all where they are
    // gathered) and an expert's weights with 32 bits.
    constexpr int64_t kMost32 = (int64_t)1 << 32;
    if (x_rows == 0 || N * ldw >= kMost32 || (gathered ? x_rows : 256) * ldx >= kMost32) return stream_kernel(gate, fp8);
    const int64_t mean = (M + E - 1) / E;
    auto pieces = [&](int64_t slots, int64_t rows) {
        return std::min<int64_t>(E, M) * ((mean + slots - 1) / slots) * ((N + rows - 1) / rows);
    };
    if (!fp8 && pieces(16, 16) <= (wide ? 1024 : 896)) return stream_kernel(gate, fp8);
    const TileSize size = mean >= 4096 && pieces(256, 256) >= 512                         ? TileSize::kHuge
                          : pieces(128, 256) >= (wide ? 512 : 256)                        ? TileSize::kLarge
                          : pieces(64, 128) >= (wide && mean < 128 ? 640 : 384)           ? TileSize::kMedium
                                                                                          : TileSize::kSmall;
    return tile_kernel(gate, fp8, wide, size);
}

int product_impl(const char *who, int64_t M, int32_t E, int64_t N, int64_t K, const void *x, int64_t ldx, int64_t x_rows,
                 const float *x_scales, int64_t ldxs, const int32_t *tokens, const void *w, int64_t ldw,
                 const float *w_scales, const int32_t *offsets, const float *bias, int32_t act, int32_t out_type, void *out,
                 int64_t ldo, float *out_scales, int64_t ldos, void *stream)
{
    constexpr int64_t kMax = std::numeric_limits<int64_t>::max();
    if (M < 0 || E < 1 || N < 1 || K < 1 || x_rows < 0) return fail(EB_ERR_INVALID, "%s: M or x_rows below 0, or E, N or K below 1", who);
    const bool exact = (act & EB_EXACT_SUMS) != 0;
    act &= ~EB_EXACT_SUMS;
    if (act != EB_ACT_NONE && act != EB_ACT_RELU && act != EB_ACT_SILU_GATE) return fail(EB_ERR_INVALID, "%s: unknown act", who);
    if (out_type != EB_F32 && out_type != EB_F16 && out_type != EB_BF16 && out_type != EB_FP8)
        return fail(EB_ERR_INVALID, "%s: unknown out_type", who);
    const bool gate = act == EB_ACT_SILU_GATE, fp8 = out_type == EB_FP8;
    if (gate && N % 2 != 0) return fail(EB_ERR_INVALID, "%s: a gate needs an even N", who);
    if (!offsets && E != 1) return fail(EB_ERR_INVALID, "%s: several experts need offsets", who);
    // E too: slot_tile counts experts up to the wave past the last in 32 bits.
    if (M > std::numeric_limits<int32_t>::max() || E > kMostSize || N > kMostSize || K > kMostSize)
        return fail(EB_ERR_UNSUPPORTED, "%s: M of 2^31 and more, or E, N or K above 2^30", who);
    if (M == 0) return EB_OK;
    if (!x || !x_scales || !w || !w_scales || !out || (fp8 && !out_scales))
        return fail(EB_ERR_INVALID, "%s: NULL x, w, out or their scales", who);
    if (!tokens && x_rows < M) return fail(EB_ERR_INVALID, "%s: x has fewer rows than M", who);
    if (ldx < K || ldw < K || ldx % 16 != 0 || ldw % 16 != 0 || (uintptr_t)x % 16 != 0 || (uintptr_t)w % 16 != 0)
        return fail(EB_ERR_INVALID, "%s: x, w, ldx and ldw must be multiples of 16 bytes, ldx and ldw at least K", who);
    const int64_t width = gate ? N / 2 : N;
    if (ldo < width || ldxs < x_rows || (fp8 && ldos < M)) return fail(EB_ERR_INVALID, "%s: ldo, ldxs or ldos too small", who);
    if (fp8 && (ldo % 16 != 0 || (uintptr_t)out % 16 != 0)) return fail(EB_ERR_INVALID, "%s: 8-bit out and ldo must be multiples of 16", who);
    if ((uintptr_t)out % element_bytes(out_type) != 0) return fail(EB_ERR_INVALID, "%s: out is not aligned to its elements", who);
    const int64_t k_blocks = (K + kBlock - 1) / kBlock, row_blocks = (width + kBlock - 1) / kBlock;
    if (ldo > kMax / 4 / M || ldos > kMax / 4 / row_blocks || ldxs > kMax / 4 / k_blocks || (x_rows > 0 && ldx > kMax / x_rows) ||
        ldw > kMax / N / E || row_blocks > kMax / 16 / E / k_blocks)
        return fail(EB_ERR_UNSUPPORTED, "%s: a buffer exceeds 2^63 bytes", who);

    ProductArgs a{};
    a.x = (const char *)x;
    a.w = (const char *)w;
    a.x_scales = x_scales;
    a.w_scales = w_scales;
    a.bias = bias;
    a.tokens = tokens;
    a.offsets = offsets;
    a.out = out;
    a.out_scales = out_scales;
    a.ldx = ldx;
    a.ldxs = ldxs;
    a.ldw = ldw;
    a.ldo = ldo;
    a.ldos = ldos;
    a.x_rows = x_rows;
    a.M = (int32_t)M;
    a.E = E;
    a.N = (int32_t)N;
    a.K = (int32_t)K;
    a.width = (int32_t)width;
    a.k_blocks = (int32_t)k_blocks;
    a.row_blocks = (int32_t)row_blocks;
    a.w_blocks = (int32_t)row_blocks * (gate ? 2 : 1);
    a.relu = act == EB_ACT_RELU;
    a.out_type = out_type;
    const int es = element_bytes(out_type);
    a.vector_out = ldo * es % 16 == 0 && (uintptr_t)out % 16 == 0;

    const KernelPlan plan = choose_kernel(M, E, N, ldx, ldw, tokens != nullptr, x_rows, gate, out_type, exact);
    a.column_tiles = (int32_t)((width + plan.columns - 1) / plan.columns);
    // At most one tile per expert is not full.
    const int64_t most_tiles = std::min<int64_t>(offsets ? M / plan.height + E : (M + plan.height - 1) / plan.height, M);
    const int64_t slot_tiles = (most_tiles + plan.band - 1) / plan.band * plan.band;
    // A launch's threads are counted in 32 bits.
    if (slot_tiles > std::numeric_limits<uint32_t>::max() / plan.threads / a.column_tiles)
        return fail(EB_ERR_UNSUPPORTED, "%s: more tiles than one launch holds", who);
    void *args[] = {&a};
    const hipError_t err = hipLaunchKernel((void *)plan.kernel, dim3((unsigned)(slot_tiles * a.column_tiles)), dim3((unsigned)plan.threads),
                                           args, 0, (hipStream_t)stream);
    return err == hipSuccess ? EB_OK : fail(EB_ERR_HIP, "%s: kernel launch failed: %s", who, hipGetErrorString(err));
}

} // namespace

extern "C" int eb_expert_product(int64_t M, int32_t E, int64_t N, int64_t K, const void *x, int64_t ldx, int64_t x_rows,
                                 const float *x_scales, int64_t ldxs, const int32_t *tokens, const void *w, int64_t ldw,
                                 const float *w_scales, const int32_t *offsets, const float *bias, int32_t act,
                                 int32_t out_type, void *out, int64_t ldo, float *out_scales, int64_t ldos, void *stream)
{
    try {
        return product_impl("eb_expert_product", M, E, N, K, x, ldx, x_rows, x_scales, ldxs, tokens, w, ldw, w_scales, offsets,
                            bias, act, out_type, out, ldo, out_scales, ldos, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_expert_product");
    }
}
