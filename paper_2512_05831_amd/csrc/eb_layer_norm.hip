// Layer norm (include/eb_train.h): eb_layer_norm.
//
//   m = mean x,  r = 1 / sqrt(mean (x - m)^2 + eps),  n = (x - m) r,  y = n w + b
//
// A row stays in registers between the two sums and the outputs, so x is read and
// y written once: bound by memory.  A wave holds up to kSteps * 512 columns, 8
// neighbours a lane and step (16 lanes are a block of 128 that shares a scale); one
// wave takes a row, or four.

#include <type_traits>

#include "eb_train.h"

namespace {

using namespace eb_train;

constexpr int kThreads = 256;
constexpr int kStride = kWave * kEach; // columns of a wave's step

struct NormArgs {
    const void *x;
    const float *weight, *bias;
    float *mean, *rstd;
    Out y, kept;
    int64_t rows, cols, ldx;
    float eps;
};

// A sum over the kWaves waves of a row, in every lane.
template <int kWaves>
__device__ __forceinline__ float sum_row(float v, float *shared, int wave)
{
    v = sum_lanes<kWave>(v);
    if constexpr (kWaves > 1) {
        __syncthreads(); // the last sum has been read
        if (threadIdx.x % kWave == 0) shared[wave] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) v += shared[i];
    }
    return v;
}

// The outputs of columns c .. c + 7, of which d is x - mean (zeros past cols).
template <bool kRagged, bool kHeld>
__device__ __forceinline__ void write8(const NormArgs &a, const float *held, int64_t row, int c, const float *d, float rstd)
{
    const int cols = (int)a.cols;
    if (c >= ((cols + kBlock - 1) & ~(kBlock - 1))) return; // whole blocks: their 16 lanes stay together
    float n[kEach], y[kEach], w[kEach], b[kEach];
    if constexpr (kHeld) {
        __builtin_memcpy(w, held + 2 * c, sizeof(w)); // a chunk's weights, then its biases
        __builtin_memcpy(b, held + 2 * c + kEach, sizeof(b));
    } else {
        if (a.weight) widen8(load_raw<kRagged>(a.weight, c, cols), w);
        if (a.bias) widen8(load_raw<kRagged>(a.bias, c, cols), b);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) n[i] = d[i] * rstd;
    if (a.kept.p) {
        // n / scale is d times one factor, as exact as d: where that can be made of d's largest
        // (not below the floor of what a factor is made of, which rstd may lift n over).
        const int most_d = most_of_block(most8(d)), most = magnitude(__int_as_float(most_d) * rstd);
        const bool least = __int_as_float(most) <= kMostFp8 * kLeastScale, small = __int_as_float(most_d) <= kMostFp8 * kLeastScale;
        if (least || small) store_fp8(a.kept, row, c, cols, n, least ? kToLeast : to_fp8(most), most);
        else store_fp8(a.kept, row, c, cols, d, to_fp8(most_d), most);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        y[i] = kHeld || a.weight ? n[i] * w[i] : n[i];
        if (kHeld || a.bias) y[i] += b[i];
    }
    store_out<kRagged>(a.y, row, c, cols, y);
}

// kSteps * 512 columns a wave; kLoop: any number of them, read again for each sum.
template <typename T, int kSteps, int kWaves, bool kLoop, bool kRagged>
__global__ __launch_bounds__(kThreads, kSteps > 4 ? 4 : 6) void eb_layer_norm_rows(NormArgs a)
{
    __shared__ float shared[kWaves];
    constexpr int kRows = kThreads / kWave / kWaves;
    const int thread_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wave = thread_wave % kWaves;
    const int64_t row = (int64_t)blockIdx.x * kRows + thread_wave / kWaves;
    if (row >= a.rows) return; // whole workgroups where waves share a row
    const T *x = (const T *)a.x + row * a.ldx;
    const int cols = (int)a.cols, first = wave * kStride + threadIdx.x % kWave * kEach;
    constexpr int kAll = kStride * kWaves;
    auto centred = [&](int c, float *f, float mean) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) f[i] -= mean;
        if (!kRagged) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) f[i] = c < cols ? f[i] : 0.f;
        } else if (c + kEach > cols) {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (c + i >= cols) f[i] = 0.f;
        }
    };
    auto add = [](const float *f, float sum) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum += f[i];
        return sum;
    };
    auto add_squares = [](const float *f, float sum) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) sum = fmaf(f[i], f[i], sum);
        return sum;
    };
    auto statistics = [&](float mean, float rstd) {
        if (threadIdx.x % (kWaves * kWave) == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    };
    const float of = (float)cols;
    float sum = 0.f, square = 0.f;
    if constexpr (kLoop) {
        float f[kEach];
        const int blocks = (cols + kBlock - 1) & ~(kBlock - 1);
        for (int c = first; c < cols; c += kAll) {
            widen8(load_raw<kRagged>(x, c, cols), f);
            sum = add(f, sum);
        }
        const float mean = sum_row<kWaves>(sum, shared, wave) / of;
        for (int c = first; c < cols; c += kAll) {
            widen8(load_raw<kRagged>(x, c, cols), f);
            centred(c, f, mean);
            square = add_squares(f, square);
        }
        const float rstd = 1.f / sqrtf(sum_row<kWaves>(square, shared, wave) / of + a.eps);
        statistics(mean, rstd);
        for (int c = first; c < blocks; c += kAll) {
            widen8(load_raw<kRagged>(x, c, cols), f);
            centred(c, f, mean);
            write8<kRagged, false>(a, nullptr, row, c, f, rstd);
        }
    } else {
        float f[kSteps][kEach];
        {
            Raw<T> raw[kSteps];
#pragma unroll
            for (int i = 0; i < kSteps; ++i) raw[i] = fetch_raw<kRagged>(x, first + i * kAll, cols);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                widen8(settle_raw<kRagged>(raw[i], first + i * kAll, cols), f[i]);
                sum = add(f[i], sum);
            }
        }
        const float mean = sum_row<kWaves>(sum, shared, wave) / of;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            centred(first + i * kAll, f[i], mean);
            square = add_squares(f[i], square);
        }
        const float rstd = 1.f / sqrtf(sum_row<kWaves>(square, shared, wave) / of + a.eps);
        statistics(mean, rstd);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            write8<kRagged, false>(a, nullptr, row, first + i * kAll, f[i], rstd);
            __builtin_amdgcn_sched_barrier(0); // not all steps' weights at a time: registers
        }
    }
}

// Many rows of up to 4096 columns with weights: a workgroup reads those once for its
// eight rows, a wave each, into LDS while the rows are on their way (else every row
// waits for its weights, step after step: 16384 x 3328 fp32 90 us, so 78.5, 4.9 TB/s).
constexpr int kHeldRows = 8;

template <typename T, int kSteps>
__global__ __launch_bounds__(kHeldRows * kWave, 4) void eb_layer_norm_held(NormArgs a)
{
    __shared__ alignas(16) float held[kSteps * kStride * 2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), cols = (int)a.cols, first = threadIdx.x % kWave * kEach;
    const int64_t row = min((int64_t)blockIdx.x * kHeldRows + wave, a.rows - 1); // past the end: the last one again
    const T *x = (const T *)a.x + row * a.ldx;
    Raw<T> raw[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) raw[i] = load_raw<false>(x, first + i * kStride, cols);
    // The chunks of weights are the waves' in turn.
#pragma unroll
    for (int i = 0; i < (kSteps + kHeldRows - 1) / kHeldRows; ++i) {
        const int c = (i * kHeldRows + wave) * kStride + first;
        if (i * kHeldRows + wave >= kSteps) break;
        float w[kEach], b[kEach] = {};
#pragma unroll
        for (int j = 0; j < kEach; ++j) w[j] = 1.f;
        if (a.weight) widen8(load_raw<false>(a.weight, c, cols), w);
        if (a.bias) widen8(load_raw<false>(a.bias, c, cols), b);
        __builtin_memcpy(held + 2 * c, w, sizeof(w));
        __builtin_memcpy(held + 2 * c + kEach, b, sizeof(b));
    }
    float f[kSteps][kEach], sum = 0.f, square = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        widen8(raw[i], f[i]);
#pragma unroll
        for (int j = 0; j < kEach; ++j) sum += f[i][j];
    }
    const float mean = sum_lanes<kWave>(sum) / (float)cols;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const bool there = first + i * kStride < cols;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            f[i][j] = there ? f[i][j] - mean : 0.f;
            square = fmaf(f[i][j], f[i][j], square);
        }
    }
    const float rstd = 1.f / sqrtf(sum_lanes<kWave>(square) / (float)cols + a.eps);
    if (threadIdx.x % kWave == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        write8<false, true>(a, held, row, first + i * kStride, f[i], rstd);
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <typename T, bool kRagged>
void *rows_kernel(int64_t cols, int *rows)
{
    *rows = cols > 8 * kStride ? 1 : 4;
    if (cols > 8 * 4 * kStride) return (void *)eb_layer_norm_rows<T, 1, 4, true, kRagged>;
    if (cols > 4 * 4 * kStride) return (void *)eb_layer_norm_rows<T, 8, 4, false, kRagged>;
    if (cols > 8 * kStride) return (void *)eb_layer_norm_rows<T, 4, 4, false, kRagged>;
    if (cols > 4 * kStride) return (void *)eb_layer_norm_rows<T, 8, 1, false, kRagged>;
    if (cols > 2 * kStride) return (void *)eb_layer_norm_rows<T, 4, 1, false, kRagged>;
    if (cols > kStride) return (void *)eb_layer_norm_rows<T, 2, 1, false, kRagged>;
    return (void *)eb_layer_norm_rows<T, 1, 1, false, kRagged>;
}

template <typename T>
void *held_kernel(int64_t cols)
{
    switch ((cols + kStride - 1) / kStride) {
    case 1: return (void *)eb_layer_norm_held<T, 1>;
    case 2: return (void *)eb_layer_norm_held<T, 2>;
    case 3: return (void *)eb_layer_norm_held<T, 3>;
    case 4: return (void *)eb_layer_norm_held<T, 4>;
    case 5: return (void *)eb_layer_norm_held<T, 5>;
    case 6: return (void *)eb_layer_norm_held<T, 6>;
    case 7: return (void *)eb_layer_norm_held<T, 7>;
    default: return (void *)eb_layer_norm_held<T, 8>;
    }
}

struct Plan {
    void *kernel;
    int64_t grid;
    int threads;
};

template <typename T>
Plan plan_of(int64_t rows, int64_t cols, bool affine)
{
    constexpr int64_t kMany = 2048;
    if (affine && cols % kEach == 0 && cols <= 8 * kStride && rows >= kMany)
        return {held_kernel<T>(cols), rows / kHeldRows + (rows % kHeldRows != 0), kHeldRows * kWave};
    int each = 1;
    void *kernel = cols % kEach ? rows_kernel<T, true>(cols, &each) : rows_kernel<T, false>(cols, &each);
    return {kernel, rows / each + (rows % each != 0), kThreads};
}

int norm_impl(const char *who, int64_t rows, int64_t cols, const void *x, int32_t dtype, int64_t ldx, const float *weight, const float *bias,
              float eps, int32_t out_type, void *y, int64_t ldy, float *y_scales, int64_t ldys, void *kept, int64_t ldk, float *kept_scales,
              int64_t ldks, float *mean, float *rstd, void *stream)
{
    if (rows < 0 || cols < 1) return fail(EB_ERR_INVALID, "%s: negative rows, or no columns", who);
    if (!floating(dtype) || (!floating(out_type) && out_type != EB_FP8)) return fail(EB_ERR_INVALID, "%s: unknown dtype or out_type", who);
    if (!(eps >= 0.f)) return fail(EB_ERR_INVALID, "%s: eps below 0", who);
    if (cols > (int64_t)1 << 30) return fail(EB_ERR_UNSUPPORTED, "%s: more than 2^30 columns", who);
    if (int rc = check_matrix(who, "x", x, dtype, rows, cols, ldx, nullptr, 0)) return rc;
    if (int rc = check_matrix(who, "y", y, out_type, rows, cols, ldy, y_scales, ldys)) return rc;
    if (kept)
        if (int rc = check_matrix(who, "kept", kept, EB_FP8, rows, cols, ldk, kept_scales, ldks)) return rc;
    if (rows == 0) return EB_OK;
    NormArgs a{};
    a.x = x;
    a.weight = weight;
    a.bias = bias;
    a.mean = mean;
    a.rstd = rstd;
    a.y = {y, y_scales, ldy, ldys, out_type};
    a.kept = {kept, kept_scales, ldk, ldks, EB_FP8};
    a.rows = rows;
    a.cols = cols;
    a.ldx = ldx;
    a.eps = eps;
    const bool affine = weight || bias;
    const Plan plan = dtype == EB_F32   ? plan_of<float>(rows, cols, affine)
                      : dtype == EB_F16 ? plan_of<_Float16>(rows, cols, affine)
                                        : plan_of<Bf16>(rows, cols, affine);
    return launch(who, plan.kernel, plan.grid, plan.threads, &a, stream);
}

} // namespace

extern "C" int eb_layer_norm(int64_t rows, int64_t cols, const void *x, int32_t dtype, int64_t ldx, const float *weight, const float *bias,
                             float eps, int32_t out_type, void *y, int64_t ldy, float *y_scales, int64_t ldys, void *kept, int64_t ldk,
                             float *kept_scales, int64_t ldks, float *mean, float *rstd, void *stream)
{
    try {
        return norm_impl("eb_layer_norm", rows, cols, x, dtype, ldx, weight, bias, eps, out_type, y, ldy, y_scales, ldys, kept, ldk,
                         kept_scales, ldks, mean, rstd, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_layer_norm");
    }
}
