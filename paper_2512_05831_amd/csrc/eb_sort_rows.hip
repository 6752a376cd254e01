// Rows sorted by expert and joined again (include/eb_train.h): eb_dispatch,
// eb_combine, eb_combine_backward.
//
//   dispatch: out[m] = x[tokens[m]]
//   combine: out[t] = sum_k w[t, k] y[slots[t, k]]
//   combine's gradients: dy[slots[t, k]] = w[t, k] dout[t], dw[t, k] = dout[t] . y[slots[t, k]]
//
// Every row is read and written once: bound by memory.  Lanes take 16 bytes (or 8
// values) of a row each, in accesses of any alignment; short rows share a wave.
// 16384 tokens, 4 of 64 experts, 1024 bf16 columns: combine 35 us (4.9 TB/s), its
// gradients to 8 bits 53 (4.5 TB/s).

#include <type_traits>

#include "eb_train.h"

namespace {

using namespace eb_train;

constexpr int kThreads = 256;

// ------------------------------------------------------------------ dispatch

struct DispatchArgs {
    const char *x;
    char *out;
    const int32_t *tokens;
    const float *x_scales;
    float *out_scales;
    int64_t M, x_rows, bytes; // bytes of a row
    int64_t ldx, ldo;         // in bytes
    int64_t ldxs, ldos, blocks;
};

constexpr int kPiece = 16;
typedef short i16_any __attribute__((aligned(1)));

// kRowLanes lanes take a row. 8192 slots, half of them used, of 1512 fp16 columns 4.3 us
// (4.3 TB/s of 18.6 MB).
template <int kRowLanes>
__global__ __launch_bounds__(kThreads) void eb_dispatch_rows(DispatchArgs a)
{
    constexpr int kRows = kThreads / kRowLanes;
    const int64_t m = (int64_t)blockIdx.x * kRows + threadIdx.x / kRowLanes;
    const int lane = threadIdx.x % kRowLanes;
    const int64_t t = m < a.M ? a.tokens[m] : -1;
    if (t >= 0 && t < a.x_rows) {
        const char *from = a.x + t * a.ldx;
        char *to = a.out + m * a.ldo;
        if (a.bytes >= kPiece) { // the last piece ends with the row, over a part of the one before
            for (int64_t c = lane * kPiece; c < a.bytes; c += kRowLanes * kPiece) {
                const int64_t at = c + kPiece <= a.bytes ? c : a.bytes - kPiece;
                *(i32x4_any *)(to + at) = *(const i32x4_any *)(from + at);
            }
        } else {
            for (int64_t c = 2 * lane; c < a.bytes; c += 2 * kRowLanes) *(i16_any *)(to + c) = *(const i16_any *)(from + c);
        }
    }
    // The rows' scales, those of a block column side by side.
    for (int64_t i = threadIdx.x; i < kRows * a.blocks; i += kThreads) {
        const int64_t row = (int64_t)blockIdx.x * kRows + i % kRows, b = i / kRows;
        const int64_t from = row < a.M ? a.tokens[row] : -1;
        if (from >= 0 && from < a.x_rows) a.out_scales[b * a.ldos + row] = a.x_scales[b * a.ldxs + from];
    }
}

// ------------------------------------------------------------------- combine

struct CombineArgs {
    const void *y, *dout;
    const int32_t *slots;
    const float *weights;
    float *dweights;
    Out out;
    int64_t N, cols, ldy, y_rows, lddout;
    int32_t K;
};

template <typename T, int kRowLanes, bool kRagged>
__global__ __launch_bounds__(kThreads) void eb_combine_rows(CombineArgs a)
{
    constexpr int kRows = kThreads / kRowLanes;
    constexpr int kAhead = 4; // pairs whose rows are on the way at a time
    const int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / kRowLanes;
    if (t >= a.N) return;
    const T *y = (const T *)a.y;
    const int32_t *slots = a.slots + t * a.K;
    const float *weights = a.weights ? a.weights + t * a.K : nullptr;
    for (int c = threadIdx.x % kRowLanes * kEach; c < a.cols; c += kRowLanes * kEach) {
        float sum[kEach] = {};
        for (int k0 = 0; k0 < a.K; k0 += kAhead) {
            Raw<T> raw[kAhead];
            float w[kAhead];
            bool there[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int64_t s = k0 + i < a.K ? slots[k0 + i] : -1;
                there[i] = s >= 0 && s < a.y_rows;
                if (there[i]) {
                    raw[i] = fetch_raw<kRagged>(y + s * a.ldy, c, a.cols);
                    w[i] = weights ? weights[k0 + i] : 1.f;
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (!there[i]) continue;
                float f[kEach];
                widen8(settle_raw<kRagged>(raw[i], c, a.cols), f);
#pragma unroll
                for (int j = 0; j < kEach; ++j) sum[j] = fmaf(w[i], f[j], sum[j]);
            }
        }
        store_out<kRagged>(a.out, t, c, (int)a.cols, sum);
    }
}

// ----------------------------------------------------------- combine's gradients

// A token's row of dout in registers, kSteps * kRowLanes * 8 columns at a time (a
// part), for all its pairs; with several parts lane k keeps the sum for pair k.
template <typename D, typename T, int kRowLanes, int kSteps, bool kRagged>
__global__ __launch_bounds__(kThreads) void eb_combine_back(CombineArgs a)
{
    constexpr int kRows = kThreads / kRowLanes;
    constexpr int kStride = kRowLanes * kEach, kPart = kStride * kSteps;
    const int cols = (int)a.cols;
    const int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / kRowLanes;
    if (t >= a.N) return;
    const int lane = threadIdx.x % kRowLanes;
    const D *dout = (const D *)a.dout + t * a.lddout;
    const bool fp8 = a.out.type == EB_FP8;
    float kept = 0.f;
    for (int part = 0; part < cols; part += kPart) {
        const int first = part + lane * kEach;
        Raw<D> raw[kSteps];
        float d[kSteps][kEach];
        int most[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) raw[i] = fetch_raw<kRagged>(dout, first + i * kStride, cols);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            widen8(settle_raw<kRagged>(raw[i], first + i * kStride, cols), d[i]);
            if (fp8) most[i] = most_of_block(most8(d[i]));
        }
        for (int k = 0; k < a.K; ++k) {
            const int64_t s = a.slots[t * a.K + k];
            if (s < 0 || s >= a.y_rows) {
                if (a.dweights && part == 0 && kPart >= cols && lane == 0) a.dweights[t * a.K + k] = 0.f;
                continue;
            }
            if (a.dweights) {
                const T *y = (const T *)a.y + s * a.ldy;
                Raw<T> other[kSteps];
#pragma unroll
                for (int i = 0; i < kSteps; ++i) other[i] = fetch_raw<kRagged>(y, first + i * kStride, cols);
                float dot = 0.f;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    float f[kEach];
                    widen8(settle_raw<kRagged>(other[i], first + i * kStride, cols), f);
#pragma unroll
                    for (int j = 0; j < kEach; ++j) dot = fmaf(d[i][j], f[j], dot);
                }
                dot = sum_lanes<kRowLanes>(dot);
                if (kPart >= cols) {
                    if (lane == 0) a.dweights[t * a.K + k] = dot;
                } else if (lane == k) { // only waves of one token have several parts
                    kept += dot;
                }
            }
            if (a.out.p) {
                const float w = a.weights ? a.weights[t * a.K + k] : 1.f;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    float f[kEach];
#pragma unroll
                    for (int j = 0; j < kEach; ++j) f[j] = w * d[i][j];
                    // A product rounds as its factor orders: the largest is the largest's.
                    const int scaled = fp8 ? magnitude(w * __int_as_float(most[i])) : 0;
                    if (fp8) store_fp8(a.out, s, first + i * kStride, cols, f, to_fp8(scaled), scaled);
                    else store_out<kRagged>(a.out, s, first + i * kStride, cols, f);
                }
            }
        }
    }
    if (kRowLanes == kWave && a.dweights && kPart < cols && lane < a.K) a.dweights[t * a.K + lane] = kept;
}

// --------------------------------------------------------------------- host

int check_sizes(const char *who, int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 1) return fail(EB_ERR_INVALID, "%s: negative rows, or no columns", who);
    if (rows > kMax32 || cols > (int64_t)1 << 30) return fail(EB_ERR_UNSUPPORTED, "%s: 2^31 rows and more, or more than 2^30 columns", who);
    return EB_OK;
}

int dispatch_impl(const char *who, int64_t M, int64_t cols, const void *x, int32_t dtype, int64_t ldx, int64_t x_rows, const float *x_scales,
                  int64_t ldxs, const int32_t *tokens, void *out, int64_t ldo, float *out_scales, int64_t ldos, void *stream)
{
    if (int rc = check_sizes(who, M, cols)) return rc;
    if (x_rows < 0) return fail(EB_ERR_INVALID, "%s: negative x_rows", who);
    if (!floating(dtype) && dtype != EB_FP8) return fail(EB_ERR_INVALID, "%s: unknown dtype", who);
    if (int rc = check_matrix(who, "x", x, dtype, x_rows, cols, ldx, x_scales, ldxs)) return rc;
    if (int rc = check_matrix(who, "out", out, dtype, M, cols, ldo, out_scales, ldos)) return rc;
    if (M > 0 && !tokens) return fail(EB_ERR_INVALID, "%s: tokens is NULL", who);
    if (M == 0 || x_rows == 0) return EB_OK;
    const int es = element_bytes(dtype);
    DispatchArgs a{};
    a.x = (const char *)x;
    a.out = (char *)out;
    a.tokens = tokens;
    a.M = M;
    a.x_rows = x_rows;
    a.bytes = dtype == EB_FP8 ? (cols + 15) & ~(int64_t)15 : cols * es;
    a.ldx = ldx * es;
    a.ldo = ldo * es;
    if (dtype == EB_FP8) {
        a.x_scales = x_scales;
        a.out_scales = out_scales;
        a.ldxs = ldxs;
        a.ldos = ldos;
        a.blocks = (cols + kBlock - 1) / kBlock;
    }
    const int64_t pieces = (a.bytes + kPiece - 1) / kPiece;
    const int lanes = pieces > 16 ? 64 : pieces > 4 ? 16 : 4;
    void *kernel = lanes == 64 ? (void *)eb_dispatch_rows<64> : lanes == 16 ? (void *)eb_dispatch_rows<16> : (void *)eb_dispatch_rows<4>;
    const int rows = kThreads / lanes;
    return launch(who, kernel, (M + rows - 1) / rows, kThreads, &a, stream);
}

template <typename T, bool kRagged>
void *combine_kernel(int lanes)
{
    return lanes == 64   ? (void *)eb_combine_rows<T, 64, kRagged>
           : lanes == 16 ? (void *)eb_combine_rows<T, 16, kRagged>
                         : (void *)eb_combine_rows<T, 4, kRagged>;
}

template <typename T>
void *combine_kernel(int lanes, bool ragged)
{
    return ragged ? combine_kernel<T, true>(lanes) : combine_kernel<T, false>(lanes);
}

int check_combine(const char *who, int64_t N, int32_t K, int64_t cols, int64_t y_rows, const int32_t *slots)
{
    if (int rc = check_sizes(who, N, cols)) return rc;
    if (K < 1 || y_rows < 0) return fail(EB_ERR_INVALID, "%s: K below 1, or negative y_rows", who);
    if (K > 64 || N > kMax32 / K) return fail(EB_ERR_UNSUPPORTED, "%s: K above 64, or 2^31 pairs and more", who);
    if (N > 0 && !slots) return fail(EB_ERR_INVALID, "%s: slots is NULL", who);
    return EB_OK;
}

int combine_impl(const char *who, int64_t N, int32_t K, int64_t cols, const void *y, int32_t y_type, int64_t ldy, int64_t y_rows,
                 const int32_t *slots, const float *weights, int32_t out_type, void *out, int64_t ldo, void *stream)
{
    if (int rc = check_combine(who, N, K, cols, y_rows, slots)) return rc;
    if (!floating(y_type) || !floating(out_type)) return fail(EB_ERR_INVALID, "%s: unknown y_type or out_type", who);
    if (int rc = check_matrix(who, "y", y, y_type, y_rows, cols, ldy, nullptr, 0)) return rc;
    if (int rc = check_matrix(who, "out", out, out_type, N, cols, ldo, nullptr, 0)) return rc;
    if (N == 0) return EB_OK;
    CombineArgs a{};
    a.y = y;
    a.slots = slots;
    a.weights = weights;
    a.out = {out, nullptr, ldo, 0, out_type};
    a.N = N;
    a.cols = cols;
    a.ldy = ldy;
    a.y_rows = y_rows;
    a.K = K;
    const int64_t pieces = (cols + kEach - 1) / kEach;
    const int lanes = pieces > 16 ? 64 : pieces > 4 ? 16 : 4, rows = kThreads / lanes;
    const bool ragged = cols % kEach != 0;
    void *kernel = y_type == EB_F32   ? combine_kernel<float>(lanes, ragged)
                   : y_type == EB_F16 ? combine_kernel<_Float16>(lanes, ragged)
                                      : combine_kernel<Bf16>(lanes, ragged);
    return launch(who, kernel, (N + rows - 1) / rows, kThreads, &a, stream);
}

template <typename D, typename T>
void *back_kernel(int64_t cols, int *rows)
{
    *rows = cols <= 128 ? kThreads / 16 : kThreads / kWave;
    if (cols % kEach) return cols <= 128 ? (void *)eb_combine_back<D, T, 16, 1, true> : (void *)eb_combine_back<D, T, 64, 2, true>;
    if (cols <= 128) return (void *)eb_combine_back<D, T, 16, 1, false>;
    if (cols <= 512) return (void *)eb_combine_back<D, T, 64, 1, false>;
    if (cols <= 1024) return (void *)eb_combine_back<D, T, 64, 2, false>;
    return (void *)eb_combine_back<D, T, 64, 4, false>;
}

template <typename D>
void *back_kernel(int32_t y_type, int64_t cols, int *rows)
{
    return y_type == EB_F32   ? back_kernel<D, float>(cols, rows)
           : y_type == EB_F16 ? back_kernel<D, _Float16>(cols, rows)
                              : back_kernel<D, Bf16>(cols, rows);
}

int back_impl(const char *who, int64_t N, int32_t K, int64_t cols, const void *dout, int32_t dout_type, int64_t lddo, const void *y,
              int32_t y_type, int64_t ldy, int64_t y_rows, const int32_t *slots, const float *weights, int32_t dy_type, void *dy,
              int64_t lddy, float *dy_scales, int64_t lddys, float *dweights, void *stream)
{
    if (int rc = check_combine(who, N, K, cols, y_rows, slots)) return rc;
    if (!floating(dout_type) || !floating(y_type) || (!floating(dy_type) && dy_type != EB_FP8))
        return fail(EB_ERR_INVALID, "%s: unknown dout_type, y_type or dy_type", who);
    if (int rc = check_matrix(who, "dout", dout, dout_type, N, cols, lddo, nullptr, 0)) return rc;
    if (dweights)
        if (int rc = check_matrix(who, "y", y, y_type, y_rows, cols, ldy, nullptr, 0)) return rc;
    if (dy)
        if (int rc = check_matrix(who, "dy", dy, dy_type, y_rows, cols, lddy, dy_scales, lddys)) return rc;
    if (N == 0 || (!dy && !dweights)) return EB_OK;
    CombineArgs a{};
    a.y = y;
    a.dout = dout;
    a.slots = slots;
    a.weights = weights;
    a.dweights = dweights;
    a.out = {dy, dy_scales, lddy, lddys, dy_type};
    a.N = N;
    a.cols = cols;
    a.ldy = ldy;
    a.y_rows = y_rows;
    a.lddout = lddo;
    a.K = K;
    int rows = 1;
    void *kernel = dout_type == EB_F32   ? back_kernel<float>(y_type, cols, &rows)
                   : dout_type == EB_F16 ? back_kernel<_Float16>(y_type, cols, &rows)
                                         : back_kernel<Bf16>(y_type, cols, &rows);
    return launch(who, kernel, (N + rows - 1) / rows, kThreads, &a, stream);
}

} // namespace

extern "C" int eb_dispatch(int64_t M, int64_t cols, const void *x, int32_t dtype, int64_t ldx, int64_t x_rows, const float *x_scales,
                           int64_t ldxs, const int32_t *tokens, void *out, int64_t ldo, float *out_scales, int64_t ldos, void *stream)
{
    try {
        return dispatch_impl("eb_dispatch", M, cols, x, dtype, ldx, x_rows, x_scales, ldxs, tokens, out, ldo, out_scales, ldos, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_dispatch");
    }
}

extern "C" int eb_combine(int64_t N, int32_t K, int64_t cols, const void *y, int32_t y_type, int64_t ldy, int64_t y_rows,
                          const int32_t *slots, const float *weights, int32_t out_type, void *out, int64_t ldo, void *stream)
{
    try {
        return combine_impl("eb_combine", N, K, cols, y, y_type, ldy, y_rows, slots, weights, out_type, out, ldo, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_combine");
    }
}

extern "C" int eb_combine_backward(int64_t N, int32_t K, int64_t cols, const void *dout, int32_t dout_type, int64_t lddo, const void *y,
                                   int32_t y_type, int64_t ldy, int64_t y_rows, const int32_t *slots, const float *weights,
                                   int32_t dy_type, void *dy, int64_t lddy, float *dy_scales, int64_t lddys, float *dweights, void *stream)
{
    try {
        return back_impl("eb_combine_backward", N, K, cols, dout, dout_type, lddo, y, y_type, ldy, y_rows, slots, weights, dy_type, dy,
                         lddy, dy_scales, lddys, dweights, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_combine_backward");
    }
}
