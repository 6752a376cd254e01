// eb_weight_gradient (include/eb_train.h): checks of arguments and the choice of
// its kernel.

#include <algorithm>

#include "eb_weight_gradient.h"

namespace {

using namespace eb_gradient;

constexpr int64_t kMostSize = (int64_t)1 << 30;

// The splits' sums added in order.
__global__ __launch_bounds__(kThreads) void eb_gradient_join(GradientArgs a)
{
    const int64_t all = (int64_t)a.E * a.N * a.K;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kThreads) {
        float v = 0.f;
        for (int s = 0; s < a.splits; ++s) v += a.partial[s * all + i];
        const int64_t place = i / a.K * a.lddw + i % a.K;
        if (a.out_type == EB_F32) {
            float *to = (float *)a.dw + place;
            *to = a.accumulate ? *to + v : v;
        } else if (a.out_type == EB_F16) {
            _Float16 *to = (_Float16 *)a.dw + place;
            *to = (_Float16)(a.accumulate ? (float)*to + v : v);
        } else {
            __bf16 *to = (__bf16 *)a.dw + place;
            *to = (__bf16)(a.accumulate ? (float)*to + v : v);
        }
    }
}

int check_sizes(const char *who, int64_t M, int32_t E, int64_t N, int64_t K)
{
    if (M < 0 || E < 1 || N < 1 || K < 1) return fail(EB_ERR_INVALID, "%s: M below 0, or E, N or K below 1", who);
    if (M > kMax32 || E > kMostSize || N > kMostSize || K > kMostSize || N * K > kMax64 / 8 / E)
        return fail(EB_ERR_UNSUPPORTED, "%s: M of 2^31 and more, or E, N, K or all weights too large", who);
    return EB_OK;
}

int64_t tiles_of(int64_t n) { return (n + kTile - 1) / kTile; }

// Parts that an expert's slots are split into where there are few tiles.
int32_t splits_of(int64_t M, int32_t E, int64_t N, int64_t K)
{
    constexpr int64_t kEnough = 512, kLeastSlots = 256, kMostSplits = 64;
    const int64_t n = tiles_of(N), k = tiles_of(K);
    if (E >= kEnough || n >= kEnough || k >= kEnough || E * n * k >= kEnough) return 1;
    const int64_t mean = (M + E - 1) / E;
    return (int32_t)std::max<int64_t>(1, std::min(std::min(kEnough / (E * n * k), mean / kLeastSlots), kMostSplits));
}

int64_t workspace_of(int64_t M, int32_t E, int64_t N, int64_t K)
{
    const int64_t splits = splits_of(M, E, N, K);
    return splits > 1 ? splits * E * N * K * 4 : 0;
}

template <typename D, typename X>
void *kernel_of(bool exact)
{
    return exact ? (void *)eb_gradient_tile<D, X, true> : (void *)eb_gradient_tile<D, X, false>;
}

template <typename D>
void *kernel_of(int32_t x_type, bool exact)
{
    return x_type == EB_FP8 ? kernel_of<D, Fp8>(exact) : x_type == EB_F16 ? kernel_of<D, _Float16>(exact) : kernel_of<D, Bf16>(exact);
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
    GradientArgs a{};
    a.dy = (const char *)dy;
    a.x = (const char *)x;
    a.dy_scales = {dy_scales, lddys};
    a.x_scales = {x_scales, ldxs};
    a.tokens = tokens;
    a.offsets = offsets;
    a.dw = dw;
    a.partial = need > 0 ? (float *)workspace : nullptr;
    a.lddy = lddy * element_bytes(dy_type);
    a.ldx = ldx * element_bytes(x_type);
    a.x_rows = x_rows;
    a.lddw = lddw;
    a.M = (int32_t)M;
    a.E = E;
    a.N = (int32_t)N;
    a.K = (int32_t)K;
    a.n_tiles = (int32_t)tiles_of(N);
    a.k_tiles = (int32_t)tiles_of(K);
    a.splits = splits_of(M, E, N, K);
    a.out_type = out_type;
    a.accumulate = accumulate != 0;
    const int64_t square = (int64_t)a.n_tiles * a.k_tiles; // below 2^46
    const int64_t grid = square > kMax32 / E / a.splits ? kMax32 : square * E * a.splits;
    const bool exact = out_type != EB_BF16;
    void *kernel = dy_type == EB_FP8   ? kernel_of<Fp8>(x_type, exact)
                   : dy_type == EB_F16 ? kernel_of<_Float16>(x_type, exact)
                                       : kernel_of<Bf16>(x_type, exact);
    if (int rc = launch(who, kernel, grid, kThreads, &a, stream)) return rc;
    if (need == 0) return EB_OK;
    const int64_t all = E * N * K;
    return launch(who, (void *)eb_gradient_join, std::min<int64_t>((all + kThreads - 1) / kThreads, 8192), kThreads, &a, stream);
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
