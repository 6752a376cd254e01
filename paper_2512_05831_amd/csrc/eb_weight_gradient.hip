// eb_weight_gradient (include/eb_train.h): checks of arguments and the choice of
// its kernel.

#include <algorithm>
#include <utility>

#include "eb_weight_gradient.h"

namespace {

using namespace eb_gradient;

constexpr int64_t kMostSize = (int64_t)1 << 30;

// The splits' sums added in order, four neighbours a thread: a workgroup takes rows of
// dw, or, where those follow each other, all of it as one (2048 x 1000 x 1512 in 4 parts
// 6.0 us; with a division for every value 7.7).
__global__ __launch_bounds__(kThreads) void eb_gradient_join(GradientArgs a)
{
    const int64_t all = (int64_t)a.E * a.N * a.K;
    const bool one = a.lddw == a.K;
    const int64_t rows = one ? 1 : (int64_t)a.E * a.N, cols = one ? all : a.K;
    const int64_t parts = one ? gridDim.x : 1, part = one ? blockIdx.x : 0;
    for (int64_t row = one ? 0 : blockIdx.x; row < rows; row += one ? 1 : gridDim.x)
        for (int64_t c = (part * kThreads + threadIdx.x) * kQuad; c < cols; c += parts * kThreads * kQuad) {
            const float *from = a.partial + row * a.K + c;
            const int left = (int)min(cols - c, (int64_t)kQuad);
            float v[kQuad] = {};
#pragma unroll 4
            for (int s = 0; s < a.splits; ++s, from += all) {
                if (left == kQuad) {
                    const i32x4_any w = *(const i32x4_any *)from;
#pragma unroll
                    for (int j = 0; j < kQuad; ++j) v[j] += __int_as_float(w[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < kQuad; ++j)
                        if (j < left) v[j] += from[j];
                }
            }
            write_values(a, row * a.lddw + c, left, v);
        }
}

int check_sizes(const char *who, int64_t M, int32_t E, int64_t N, int64_t K)
{
    if (M < 0 || E < 1 || N < 1 || K < 1) return fail(EB_ERR_INVALID, "%s: M below 0, or E, N or K below 1", who);
    if (M > kMax32 || E > kMostSize || N > kMostSize || K > kMostSize || N * K > kMax64 / 8 / E)
        return fail(EB_ERR_UNSUPPORTED, "%s: M of 2^31 and more, or E, N, K or all weights too large", who);
    return EB_OK;
}

int64_t tiles_of(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }

// How a call is cut up, from its sizes alone (so that its workspace is known without
// types; tiles are counted with dy as the own operand: where x is that one and N small they
// are fewer, of 32 x 1024 4 and not 16, and fill less of the GPU).
// Measured in turn, us a call:
//   Shared columns 64 or 128.  Narrow tiles let three workgroups share a compute unit,
//   wide ones read less: one expert, 2048 slots by 1000 x 1512 in bf16 (1536 steps of 64
//   slots in all) 28.8 and 29.5; 32 experts of 512 x 1024, 256 slots each, to bf16 (2048) 38.0
//   and 41.7; 16384 by 512 x 512 in bf16 (2048) 32.8 and 39.4; 8192 by 1024 x 1024 in 8 bits (4096)
//   55.2 and 54.8; 2048 by 2560 x 2048 (5120) 68.8 and 65.2; 16384 by 2048 x 2048 (32768) 300 and 250.
//   Parts of an expert's slots.  They fill the GPU, and cost 8 bytes of traffic an
//   output each: 2048 slots by 1000 x 1512 in 2, 4, 8 parts 31.6, 28.8, 32.2; 8192 by 1024 x 1024
//   in 4, 8, 16 parts 70.9, 55.2, 61.6; 16384 by 2048 x 2048 in 2, 4, 8 parts 309, 250, 273.
struct Cut {
    bool narrow;
    int32_t splits;
};

Cut cut_of(int64_t M, int32_t E, int64_t N, int64_t K)
{
    constexpr int64_t kFewSteps = 4096, kWide = 512, kNarrow = 768, kLeastSlots = 512, kMostSplits = 64;
    const int64_t n = tiles_of(N, kOwnTile), mean = (M + E - 1) / E;
    auto tiles = [&](int64_t width) { // or `many`, whatever lies above
        constexpr int64_t many = (int64_t)1 << 20;
        const int64_t k = tiles_of(K, width);
        return E >= many || n >= many || k >= many || n * k >= many ? many : std::min(E * n * k, many);
    };
    Cut c{};
    c.narrow = tiles(128) * ((mean + 63) / 64) <= kFewSteps;
    c.splits = (int32_t)std::max<int64_t>(1, std::min({c.narrow ? kNarrow / tiles(64) : kWide / tiles(128), mean / kLeastSlots, kMostSplits}));
    return c;
}

int64_t workspace_of(int64_t M, int32_t E, int64_t N, int64_t K)
{
    const int64_t splits = cut_of(M, E, N, K).splits;
    return splits > 1 ? splits * E * N * K * 4 : 0;
}

int gradient_impl(const char *who, int64_t M, int32_t E, int64_t N, int64_t K, const void *dy, int32_t dy_type, int64_t lddy,
                  const float *dy_scales, int64_t lddys, const void *x, int32_t x_type, int64_t ldx, int64_t x_rows, const float *x_scales,
                  int64_t ldxs, const int32_t *tokens, const int32_t *offsets, int32_t out_type, int32_t accumulate, void *dw, int64_t lddw,
                  void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = check_sizes(who, M, E, N, K)) return rc;
    auto operand = [](int32_t type) { return type == EB_F16 || type == EB_BF16 || type == EB_FP8; };
    if (!operand(dy_type) || !operand(x_type) || !floating(out_type)) return fail(EB_ERR_INVALID, "%s: unknown dy_type, x_type or out_type", who);
    if (x_rows < 0 || (!tokens && x_rows < M)) return fail(EB_ERR_INVALID, "%s: x has fewer rows than M", who);
    if (accumulate != 0 && accumulate != 1) return fail(EB_ERR_INVALID, "%s: accumulate must be 0 or 1", who);
    if (!offsets && E != 1) return fail(EB_ERR_INVALID, "%s: several experts need offsets", who);
    if (int rc = check_matrix(who, "dy", dy, dy_type, M, N, lddy, dy_scales, lddys)) return rc;
    if (int rc = check_matrix(who, "x", x, x_type, x_rows, K, ldx, x_scales, ldxs)) return rc;
    if (int rc = check_matrix(who, "dw", dw, out_type, E * N, K, lddw, nullptr, 0)) return rc;
    const int64_t need = workspace_of(M, E, N, K);
    if (need > 0 && (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < (size_t)need))
        return fail(EB_ERR_INVALID, "%s: workspace too small or not a multiple of 16 bytes", who);
    const bool exact = out_type != EB_BF16;
    auto whole = [](const void *p, int32_t type, int64_t cols, int64_t ld) { // rows of whole pieces of 16 bytes
        return type == EB_FP8 || ((uintptr_t)p % 16 == 0 && cols % 8 == 0 && ld % 8 == 0);
    };
    const bool direct = whole(dy, dy_type, N, lddy) && whole(x, x_type, K, ldx);
    const auto [few, splits] = cut_of(M, E, N, K);
    const bool narrow = few || !direct;
    const Choice choice = dy_type == EB_FP8   ? choice_fp8(x_type, exact, direct, narrow)
                          : dy_type == EB_F16 ? choice_f16(x_type, exact, direct, narrow)
                                              : choice_bf16(x_type, exact, direct, narrow);
    GradientArgs a{};
    a.own = (const char *)dy;
    a.shared = (const char *)x;
    a.own_scales = {dy_scales, lddys};
    a.shared_scales = {x_scales, ldxs};
    a.own_ld = lddy * element_bytes(dy_type);
    a.shared_ld = ldx * element_bytes(x_type);
    a.own_cols = (int32_t)N;
    a.shared_cols = (int32_t)K;
    if (choice.own_x) {
        std::swap(a.own, a.shared);
        std::swap(a.own_scales, a.shared_scales);
        std::swap(a.own_ld, a.shared_ld);
        std::swap(a.own_cols, a.shared_cols);
    }
    a.tokens = tokens;
    a.offsets = offsets;
    a.dw = dw;
    a.partial = need > 0 ? (float *)workspace : nullptr;
    a.x_rows = x_rows;
    a.lddw = lddw;
    a.M = (int32_t)M;
    a.E = E;
    a.N = (int32_t)N;
    a.K = (int32_t)K;
    a.own_tiles = (int32_t)tiles_of(a.own_cols, kOwnTile);
    a.shared_tiles = (int32_t)tiles_of(a.shared_cols, narrow ? 64 : 128);
    a.splits = splits;
    a.out_type = out_type;
    a.accumulate = accumulate != 0;
    const int64_t square = (int64_t)a.own_tiles * a.shared_tiles; // below 2^46
    const int64_t grid = square > kMax32 / E / a.splits ? kMax32 : square * E * a.splits;
    if (int rc = launch(who, choice.kernel, grid, kThreads, &a, stream)) return rc;
    if (need == 0) return EB_OK;
    const int64_t groups = lddw == K ? (E * N * K + kThreads * kQuad - 1) / (kThreads * kQuad) : E * N;
    return launch(who, (void *)eb_gradient_join, std::min<int64_t>(groups, 8192), kThreads, &a, stream);
}

int workspace_impl(const char *who, int64_t M, int32_t E, int64_t N, int64_t K, size_t *bytes)
{
    if (!bytes) return fail(EB_ERR_INVALID, "%s: bytes is NULL", who);
    if (int rc = check_sizes(who, M, E, N, K)) return rc;
    *bytes = (size_t)workspace_of(M, E, N, K);
    return EB_OK;
}

} // namespace

extern "C" int eb_weight_gradient_workspace(int64_t M, int32_t E, int64_t N, int64_t K, size_t *bytes)
{
    try {
        return workspace_impl("eb_weight_gradient_workspace", M, E, N, K, bytes);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_weight_gradient_workspace");
    }
}

extern "C" int eb_weight_gradient(int64_t M, int32_t E, int64_t N, int64_t K, const void *dy, int32_t dy_type, int64_t lddy,
                                  const float *dy_scales, int64_t lddys, const void *x, int32_t x_type, int64_t ldx, int64_t x_rows,
                                  const float *x_scales, int64_t ldxs, const int32_t *tokens, const int32_t *offsets, int32_t out_type,
                                  int32_t accumulate, void *dw, int64_t lddw, void *workspace, size_t workspace_bytes, void *stream)
{
    try {
        return gradient_impl("eb_weight_gradient", M, E, N, K, dy, dy_type, lddy, dy_scales, lddys, x, x_type, ldx, x_rows, x_scales, ldxs,
                             tokens, offsets, out_type, accumulate, dw, lddw, workspace, workspace_bytes, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_weight_gradient");
    }
}
