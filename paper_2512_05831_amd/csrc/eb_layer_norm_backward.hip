// The gradients of layer norm (include/eb_train.h): eb_layer_norm_backward.
//
//   n = (x - m) r, or as kept in 8 bits;  g = dy w
//   dx = r (g - mean g - n mean(g n)),  dweight = sum dy n,  dbias = sum dy
//
// One pass over dy and x: a row stays in registers between its two sums and dx, and
// the lanes that hold a column add its share of dweight and dbias over the rows of
// their workgroup.  The workgroups' sums wait in the workspace; a second kernel adds
// them in order, so equal calls give equal bits.  Bound by memory: 16384 x 3328 in bf16
// from 8 bits 67 us and 5 for the second kernel (4.1 TB/s), fp32 from fp32 133 (4.9 TB/s).

#include <algorithm>
#include <type_traits>

#include "eb_train.h"

namespace {

using namespace eb_train;

constexpr int kThreads = 256;
constexpr int kStride = kWave * kEach; // columns of a wave's step
constexpr int kMostGroups = 768;       // workgroups that add up dweight and dbias

struct NormBackArgs {
    const void *dy, *x;
    Scales x_scales;
    const float *mean, *rstd, *weight;
    void *dx;
    float *partial; // [workgroups][2][cols], or NULL
    int64_t rows, cols, lddy, ldx, lddx;
    int32_t dy_type;
};

template <int kWaves>
__device__ __forceinline__ float2 sum_row(float2 v, float2 *shared, int wave)
{
    v.x = sum_lanes<kWave>(v.x);
    v.y = sum_lanes<kWave>(v.y);
    if constexpr (kWaves > 1) {
        if (threadIdx.x % kWave == 0) shared[wave] = v;
        __syncthreads();
        v = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            v.x += shared[i].x;
            v.y += shared[i].y;
        }
    }
    return v;
}

template <typename D>
constexpr int kTypeOf = sizeof(D) == 4 ? EB_F32 : std::is_same_v<D, Bf16> ? EB_BF16 : EB_F16;

// A row's values as they lie in memory.
template <typename D, typename T, int kSteps>
struct RawRow {
    Raw<D> dy[kSteps];
    Raw<T> x[kSteps];
    float scale[kSteps]; // of x in 8 bits
    float rstd, mean;
};

template <typename D, typename T, int kSteps, int kWaves, bool kRagged>
__global__ __launch_bounds__(kWaves > 4 ? kWaves * kWave : kThreads) void eb_layer_norm_back(NormBackArgs a)
{
    constexpr int kRows = kWaves > 4 ? 1 : kThreads / kWave / kWaves; // rows that a workgroup holds at a time
    constexpr int kAll = kStride * kWaves;
    constexpr bool kFp8 = sizeof(T) == 1;
    __shared__ float2 shared[2][kWaves];
    __shared__ float joined[kRows > 1 ? (kRows - 1) * kSteps * kAll : 1];
    const int thread_wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wave = thread_wave % kWaves, of = thread_wave / kWaves;
    const int cols = (int)a.cols, first = wave * kStride + threadIdx.x % kWave * kEach;
    const float by = 1.f / (float)a.cols;
    float dw[kSteps][kEach] = {}, db[kSteps][kEach] = {}, w[kSteps][kEach];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (a.weight) widen8(load_raw<kRagged>(a.weight, first + i * kAll, cols), w[i]);
        else
#pragma unroll
            for (int j = 0; j < kEach; ++j) w[i][j] = 1.f;
    }
    auto load = [&](int64_t row) {
        RawRow<D, T, kSteps> r;
        const D *dy = (const D *)a.dy + row * a.lddy;
        const T *x = (const T *)a.x + row * a.ldx;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int c = first + i * kAll;
            r.dy[i] = fetch_raw<kRagged>(dy, c, cols);
            r.x[i] = fetch_raw<kRagged>(x, c, cols);
            if constexpr (kFp8) r.scale[i] = a.x_scales.p[(c < cols ? c / kBlock : 0) * a.x_scales.ld + row];
        }
        r.rstd = a.rstd[row];
        r.mean = kFp8 ? 0.f : a.mean[row];
        return r;
    };
    int turn = 0;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + of;
    RawRow<D, T, kSteps> next;
    if (row < a.rows) next = load(row);
    for (; row < a.rows; row += step, turn ^= 1) {
        const RawRow<D, T, kSteps> now = next;
        if (row + step < a.rows) next = load(row + step); // on its way while this one is worked on
        float g[kSteps][kEach], n[kSteps][kEach];
        float2 sums = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int c = first + i * kAll;
            widen8(settle_raw<kRagged>(now.dy[i], c, cols), g[i]);
            widen8(settle_raw<kRagged>(now.x[i], c, cols), n[i]);
            const float scale = kFp8 && c < cols ? now.scale[i] : 0.f;
#pragma unroll
            for (int j = 0; j < kEach; ++j) n[i][j] = kFp8 ? n[i][j] * scale : (n[i][j] - now.mean) * now.rstd;
            if (!kFp8 && !kRagged) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) n[i][j] = c < cols ? n[i][j] : 0.f;
            } else if (!kFp8 && c + kEach > cols) {
#pragma unroll
                for (int j = 0; j < kEach; ++j)
                    if (c + j >= cols) n[i][j] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                dw[i][j] = fmaf(g[i][j], n[i][j], dw[i][j]);
                db[i][j] += g[i][j];
                g[i][j] *= w[i][j];
                sums.x += g[i][j];
                sums.y = fmaf(g[i][j], n[i][j], sums.y);
            }
        }
        sums = sum_row<kWaves>(sums, shared[turn], wave);
        const float c1 = sums.x * by, c2 = sums.y * by;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int c = first + i * kAll;
            if (c >= cols) break;
            float d[kEach];
#pragma unroll
            for (int j = 0; j < kEach; ++j) d[j] = now.rstd * (g[i][j] - c1 - n[i][j] * c2);
            store8<kRagged>((D *)a.dx + row * a.lddx, kTypeOf<D>, c, cols, d);
        }
    }
    if (!a.partial) return;
    // The workgroup's rows joined, in order, then written.
    auto join = [&](float (&v)[kSteps][kEach]) {
        if constexpr (kRows > 1) {
            __syncthreads();
            if (of > 0) {
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
#pragma unroll
                    for (int j = 0; j < kEach; ++j) joined[((of - 1) * kSteps + i) * kAll + j * kWave + threadIdx.x % kWave] = v[i][j];
            }
            __syncthreads();
            if (of == 0) {
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
#pragma unroll
                    for (int j = 0; j < kEach; ++j)
#pragma unroll
                        for (int k = 0; k < kRows - 1; ++k) v[i][j] += joined[(k * kSteps + i) * kAll + j * kWave + threadIdx.x % kWave];
            }
        }
    };
    join(dw);
    join(db);
    if (of > 0) return;
    float *to = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int c = first + i * kAll;
        if (c >= cols) break;
        store8<kRagged>(to, EB_F32, c, cols, dw[i]);
        store8<kRagged>(to + a.cols, EB_F32, c, cols, db[i]);
    }
}

// Rows that registers do not hold: dy and x are read twice for dx,
template <typename D, typename T>
__device__ __forceinline__ void long_values(const NormBackArgs &a, int64_t row, int c, float r, float m, float *d, float *n)
{
    widen8(load_raw<true>((const D *)a.dy + row * a.lddy, c, a.cols), d);
    widen8(load_raw<true>((const T *)a.x + row * a.ldx, c, a.cols), n);
    const float s = sizeof(T) == 1 ? a.x_scales.p[c / kBlock * a.x_scales.ld + row] : 0.f;
#pragma unroll
    for (int j = 0; j < kEach; ++j) n[j] = sizeof(T) == 1 ? n[j] * s : c + j < a.cols ? (n[j] - m) * r : 0.f;
}

template <typename D, typename T>
__global__ __launch_bounds__(kThreads) void eb_layer_norm_back_long(NormBackArgs a)
{
    constexpr int kWaves = kThreads / kWave;
    __shared__ float2 shared[kWaves];
    const int64_t row = blockIdx.x;
    const float r = a.rstd[row], m = sizeof(T) == 1 ? 0.f : a.mean[row];
    float2 sums = {0.f, 0.f};
    float d[kEach], n[kEach], w[kEach];
    for (int c = threadIdx.x * kEach; c < a.cols; c += kThreads * kEach) {
        long_values<D, T>(a, row, c, r, m, d, n);
        if (a.weight) widen8(load_raw<true>(a.weight, c, a.cols), w);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const float g = a.weight ? d[j] * w[j] : d[j];
            sums.x += g;
            sums.y = fmaf(g, n[j], sums.y);
        }
    }
    sums = sum_row<kWaves>(sums, shared, threadIdx.x / kWave);
    const float c1 = sums.x / (float)a.cols, c2 = sums.y / (float)a.cols;
    for (int c = threadIdx.x * kEach; c < a.cols; c += kThreads * kEach) {
        long_values<D, T>(a, row, c, r, m, d, n);
        if (a.weight) widen8(load_raw<true>(a.weight, c, a.cols), w);
#pragma unroll
        for (int j = 0; j < kEach; ++j) d[j] = r * ((a.weight ? d[j] * w[j] : d[j]) - c1 - n[j] * c2);
        store8<true>((D *)a.dx + row * a.lddx, kTypeOf<D>, c, a.cols, d);
    }
}

// and once more for dweight and dbias: a workgroup takes 2048 columns of the rows
// that are its own modulo gridDim / strips.
template <typename D, typename T>
__global__ __launch_bounds__(kThreads) void eb_layer_norm_back_columns(NormBackArgs a)
{
    const int64_t strips = (a.cols + kThreads * kEach - 1) / (kThreads * kEach);
    const int c = (int)(blockIdx.x % strips * kThreads + threadIdx.x) * kEach;
    const int64_t part = blockIdx.x / strips, parts = gridDim.x / strips;
    if (c >= a.cols) return;
    float dw[kEach] = {}, db[kEach] = {};
    for (int64_t row = part; row < a.rows; row += parts) {
        float d[kEach], n[kEach];
        long_values<D, T>(a, row, c, a.rstd[row], sizeof(T) == 1 ? 0.f : a.mean[row], d, n);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            dw[j] = fmaf(d[j], n[j], dw[j]);
            db[j] += d[j];
        }
    }
    float *to = a.partial + part * 2 * a.cols;
    store8<true>(to, EB_F32, c, a.cols, dw);
    store8<true>(to + a.cols, EB_F32, c, a.cols, db);
}

// The workgroups' sums added: 64 columns of dweight and dbias side by side, 16 waves a
// share of the workgroups each.
struct JoinArgs {
    const float *partial;
    float *dweight, *dbias;
    int64_t cols;
    int32_t parts;
};

constexpr int kJoinThreads = 1024;

__global__ __launch_bounds__(kJoinThreads) void eb_layer_norm_join(JoinArgs a)
{
    __shared__ float shared[kJoinThreads];
    constexpr int kWaves = kJoinThreads / kWave;
    const int wave = threadIdx.x / kWave;
    for (int64_t first = (int64_t)blockIdx.x * kWave; first < 2 * a.cols; first += (int64_t)gridDim.x * kWave) {
        const int64_t c = first + threadIdx.x % kWave;
        float sum = 0.f;
        if (c < 2 * a.cols) {
#pragma unroll 8
            for (int p = wave; p < a.parts; p += kWaves) sum += a.partial[(int64_t)p * 2 * a.cols + c];
        }
        __syncthreads(); // the last columns' have been read
        shared[threadIdx.x] = sum;
        __syncthreads();
        if (wave > 0 || c >= 2 * a.cols) continue;
#pragma unroll
        for (int i = 1; i < kWaves; ++i) sum += shared[i * kWave + threadIdx.x];
        if (c < a.cols) {
            if (a.dweight) a.dweight[c] = sum;
        } else if (a.dbias) {
            a.dbias[c - a.cols] = sum;
        }
    }
}

constexpr int64_t kMostHeld = 2 * 8 * kStride; // columns of a row in registers

int64_t groups_of(int64_t rows, int64_t cols)
{
    if (cols > kMostHeld) {
        const int64_t strips = (cols + kThreads * kEach - 1) / (kThreads * kEach);
        return std::min<int64_t>(std::max<int64_t>(1, kMostGroups / strips), (rows + 7) / 8);
    }
    // Every workgroup leaves sums of all columns: as many as fill the GPU, then one for
    // each eight rows (2048 x 1512 fp16: 256 workgroups 15.2 us with the joining, 768 16.4).
    const int64_t held = cols > 2 * kStride ? 1 : 4, most = cols > 8 * kStride ? 384 : kMostGroups;
    return std::min({most, std::max<int64_t>(256, rows / 8), (rows + held - 1) / held});
}

struct RowPlan {
    void *kernel;
    int threads;
};

template <typename D, typename T>
RowPlan plan_of(int64_t cols)
{
    const bool ragged = cols % kEach != 0;
    if (cols > 2 * 4 * kStride) return {ragged ? (void *)eb_layer_norm_back<D, T, 2, 8, true> : (void *)eb_layer_norm_back<D, T, 2, 8, false>, 512};
    if (cols > 4 * kStride) return {ragged ? (void *)eb_layer_norm_back<D, T, 2, 4, true> : (void *)eb_layer_norm_back<D, T, 2, 4, false>, kThreads};
    if (cols > 2 * kStride) return {ragged ? (void *)eb_layer_norm_back<D, T, 1, 4, true> : (void *)eb_layer_norm_back<D, T, 1, 4, false>, kThreads};
    if (cols > kStride || ragged) return {ragged ? (void *)eb_layer_norm_back<D, T, 2, 1, true> : (void *)eb_layer_norm_back<D, T, 2, 1, false>, kThreads};
    return {(void *)eb_layer_norm_back<D, T, 1, 1, false>, kThreads};
}

template <typename D, typename T>
int run(const char *who, NormBackArgs &a, int64_t groups, void *stream)
{
    if (a.cols <= kMostHeld) {
        const RowPlan plan = plan_of<D, T>(a.cols);
        return launch(who, plan.kernel, groups, plan.threads, &a, stream);
    }
    if (int rc = launch(who, (void *)eb_layer_norm_back_long<D, T>, a.rows, kThreads, &a, stream)) return rc;
    if (!a.partial) return EB_OK;
    const int64_t strips = (a.cols + kThreads * kEach - 1) / (kThreads * kEach);
    return launch(who, (void *)eb_layer_norm_back_columns<D, T>, groups * strips, kThreads, &a, stream);
}

template <typename D>
int run(const char *who, int32_t x_type, NormBackArgs &a, int64_t groups, void *stream)
{
    if (x_type == EB_FP8) return run<D, Fp8>(who, a, groups, stream);
    if (x_type == EB_F32) return run<D, float>(who, a, groups, stream);
    if (x_type == EB_F16) return run<D, _Float16>(who, a, groups, stream);
    return run<D, Bf16>(who, a, groups, stream);
}

int check_sizes(const char *who, int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 1) return fail(EB_ERR_INVALID, "%s: negative rows, or no columns", who);
    if (cols > (int64_t)1 << 30) return fail(EB_ERR_UNSUPPORTED, "%s: more than 2^30 columns", who);
    if (rows > std::numeric_limits<uint32_t>::max() / kThreads) return fail(EB_ERR_UNSUPPORTED, "%s: more rows than one launch holds", who);
    return EB_OK;
}

int back_impl(const char *who, int64_t rows, int64_t cols, const void *dy, int32_t dy_type, int64_t lddy, const void *x, int32_t x_type,
              int64_t ldx, const float *x_scales, int64_t ldxs, const float *mean, const float *rstd, const float *weight, void *dx,
              int64_t lddx, float *dweight, float *dbias, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = check_sizes(who, rows, cols)) return rc;
    if (!floating(dy_type) || (!floating(x_type) && x_type != EB_FP8)) return fail(EB_ERR_INVALID, "%s: unknown dy_type or x_type", who);
    if (int rc = check_matrix(who, "dy", dy, dy_type, rows, cols, lddy, nullptr, 0)) return rc;
    if (int rc = check_matrix(who, "x", x, x_type, rows, cols, ldx, x_scales, ldxs)) return rc;
    if (int rc = check_matrix(who, "dx", dx, dy_type, rows, cols, lddx, nullptr, 0)) return rc;
    if (rows > 0 && (!rstd || (x_type == EB_FP8) != !mean))
        return fail(EB_ERR_INVALID, "%s: rstd is NULL, or mean is without an x in floating point or the other way round", who);
    const bool sums = dweight || dbias;
    const int64_t groups = groups_of(rows, cols);
    if (sums && rows > 0 && (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes / 8 / (size_t)cols < (size_t)groups))
        return fail(EB_ERR_INVALID, "%s: workspace too small or not a multiple of 16 bytes", who);
    NormBackArgs a{};
    a.dy = dy;
    a.x = x;
    a.x_scales = {x_scales, ldxs};
    a.mean = mean;
    a.rstd = rstd;
    a.weight = weight;
    a.dx = dx;
    a.partial = sums ? (float *)workspace : nullptr;
    a.rows = rows;
    a.cols = cols;
    a.lddy = lddy;
    a.ldx = ldx;
    a.lddx = lddx;
    a.dy_type = dy_type;
    if (rows > 0) {
        const int rc = dy_type == EB_F32   ? run<float>(who, x_type, a, groups, stream)
                       : dy_type == EB_F16 ? run<_Float16>(who, x_type, a, groups, stream)
                                           : run<Bf16>(who, x_type, a, groups, stream);
        if (rc || !sums) return rc;
    } else if (!sums) {
        return EB_OK;
    }
    JoinArgs j{(const float *)workspace, dweight, dbias, cols, (int32_t)groups};
    // In turns where they are more than a launch's threads hold: its work is under way by now.
    constexpr int64_t kMostJoins = 1 << 16;
    return launch(who, (void *)eb_layer_norm_join, std::min((2 * cols + kWave - 1) / kWave, kMostJoins), kJoinThreads, &j, stream);
}

int workspace_impl(const char *who, int64_t rows, int64_t cols, size_t *bytes)
{
    if (!bytes) return fail(EB_ERR_INVALID, "%s: bytes is NULL", who);
    if (int rc = check_sizes(who, rows, cols)) return rc;
    *bytes = (size_t)groups_of(rows, cols) * 2 * 4 * (size_t)cols;
    return EB_OK;
}

} // namespace

extern "C" int eb_layer_norm_backward_workspace(int64_t rows, int64_t cols, size_t *bytes)
{
    try {
        return workspace_impl("eb_layer_norm_backward_workspace", rows, cols, bytes);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_layer_norm_backward_workspace");
    }
}

extern "C" int eb_layer_norm_backward(int64_t rows, int64_t cols, const void *dy, int32_t dy_type, int64_t lddy, const void *x,
                                      int32_t x_type, int64_t ldx, const float *x_scales, int64_t ldxs, const float *mean,
                                      const float *rstd, const float *weight, void *dx, int64_t lddx, float *dweight, float *dbias,
                                      void *workspace, size_t workspace_bytes, void *stream)
{
    try {
        return back_impl("eb_layer_norm_backward", rows, cols, dy, dy_type, lddy, x, x_type, ldx, x_scales, ldxs, mean, rstd, weight, dx,
                         lddx, dweight, dbias, workspace, workspace_bytes, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_layer_norm_backward");
    }
}
