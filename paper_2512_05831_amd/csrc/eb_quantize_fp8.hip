// Values to 8-bit floating point with block scales: eb_quantize_fp8
// (include/eb_experts.h).
//
//   scale = max(max|x| / 448, 2^-126) in fp32,  q = e4m3(x / the same, exact)
//
// One read of x, one write of q and the scales: bound by memory.  16384 x 3328
// fp32 values in 50.7 us, 5.4 TB/s (a copy of 218 MB: 5.2), in 40 where the last level
// of cache holds some; 2048 x 1024 in 4.8, and in 3.2.
//
// 1 x 128 blocks: 16 lanes hold a block, 8 values each, so a lane writes 8
// bytes of q.  A workgroup takes 16 rows and up to kSteps blocks along them:
// the 16 scales of a block column are neighbours in memory and are written
// together.  One, two, four and eight blocks: 41.2, 40.7, 43.0 and 49.2 us.
// 128 x 128 blocks: a workgroup holds a block in registers, 64 values a lane.

#include <hip/hip_runtime.h>

#include <stdint.h>

#include <limits>
#include <type_traits>

#include "../../include/eb.h"
#include "../../include/eb_experts.h"
#include "eb_experts.h"
#include "eb_internal.h"

namespace {

using namespace eb_experts;
using eb_detail::fail;

constexpr int kThreads = 256;
constexpr int kLanes = 16;               // lanes of a 1 x 128 block
constexpr int kEach = kBlock / kLanes;   // values of a lane
constexpr int kRows = kThreads / kLanes; // rows of a workgroup
constexpr int kSteps = 2;                // block columns of a workgroup

struct QuantizeArgs {
    const void *x;
    void *q;
    float *scales;
    int64_t ldx, ldq, lds;
    int64_t rows;           // of all matrices (1 x 128), of one (128 x 128)
    int64_t cols, padded;   // padded: cols up to the next multiple of 16
    int64_t row_blocks, col_blocks;
};

// Eight values from column c of a row; zeros past cols.
template <typename T, bool kAligned>
__device__ __forceinline__ void load8(const T *row, int64_t c, int64_t cols, float *f)
{
    if (kAligned && c + kEach <= cols) {
        T v[kEach];
        constexpr int n = sizeof(v) / 16;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const i32x4 w = *(const i32x4 *)((const char *)(row + c) + 16 * i);
            __builtin_memcpy((char *)v + 16 * i, &w, 16);
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) f[i] = widen(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) f[i] = c + i < cols ? widen(row[c + i]) : 0.f;
    }
}

__device__ __forceinline__ int most8(const float *f)
{
    int m = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) m = max(m, magnitude(f[i]));
    return m;
}

// How the values of a block are brought to e4m3.
struct Steps {
    float scale;
    float lo, hi; // 448 / most, 2^-21 of it less and more
    float most;   // the largest magnitude that the scale stands for
};

__device__ __forceinline__ Steps steps_of(int most)
{
    constexpr float kLeastMost = kMostFp8 * kLeastScale;
    Steps s;
    s.scale = block_scale(most);
    s.most = fmaxf(__int_as_float(most), kLeastMost);
    const float f = kMostFp8 / s.most;
    s.lo = f * (1.f - 0x1p-21f);
    s.hi = f * (1.f + 0x1p-21f);
    return s;
}

// Four values: x * 448 / most, rounded once.  A product with lo is below the
// exact quotient, one with hi above.  Where both round alike, that is the answer;
// else (four fp32 values in a million, and ties, which are two in a thousand of
// 16-bit values) the exact quotient lies by the middle m of two e4m3 numbers, and
// |x| * 448 is compared with m * most, both over 2^9, which 64 bits hold, and
// 32 where x has 16.  (For all values two exact divisions: 50 us for 44 in blocks of
// 16384 x 3328 fp32, and 1 in 10^6 rounded otherwise.)
template <typename T>
__device__ __forceinline__ int round4(const float *f, const Steps &s)
{
    int lo = pack_fp8(f[0] * s.lo, f[1] * s.lo, f[2] * s.lo, f[3] * s.lo);
    const int hi = pack_fp8(f[0] * s.hi, f[1] * s.hi, f[2] * s.hi, f[3] * s.hi);
    if (__any(lo != hi)) {
        auto settle = [&](auto at) {
            constexpr int i = decltype(at)::value, kByte = (int)(0xFFu << 8 * i);
            using Exact = std::conditional_t<sizeof(T) == 4, double, float>;
            const Exact x = (Exact)fabsf(f[i]) * (Exact)(kMostFp8 * 0x1p-9f);
            const float a = __builtin_amdgcn_cvt_f32_fp8(lo, i), b = __builtin_amdgcn_cvt_f32_fp8(hi, i);
            const Exact m = (Exact)(fabsf(a + b) * 0x1p-10f) * (Exact)s.most;
            const bool up = x > m || (x == m && (lo >> 8 * i & 1));
            if (((lo ^ hi) & kByte) && up) lo = (lo & ~kByte) | (hi & kByte);
        };
        settle(std::integral_constant<int, 0>());
        settle(std::integral_constant<int, 1>());
        settle(std::integral_constant<int, 2>());
        settle(std::integral_constant<int, 3>());
    }
    return lo;
}

// Their e4m3 values to column c of q, where the row (with its padding) has it;
// `left`: how many of the columns there are.
template <typename T>
__device__ __forceinline__ void store8(char *row, int64_t c, int64_t padded, int left, const float *f, const Steps &s)
{
    int2 v;
    v.x = round4<T>(f, s);
    v.y = round4<T>(f + 4, s);
    if (!(s.scale == s.scale)) { // only NaNs, but for the padding
        const uint64_t all = 0x7F7F7F7F7F7F7F7Full, some = left >= 8 ? all : left <= 0 ? 0 : all >> 8 * (8 - left);
        v.x = (int)some;
        v.y = (int)(some >> 32);
    }
    if (c < padded) *(int2 *)(row + c) = v;
}

template <typename T, bool kAligned>
__global__ __launch_bounds__(kThreads) void eb_quantize_rows(QuantizeArgs a)
{
    const int64_t strips = (a.col_blocks + kSteps - 1) / kSteps;
    const int64_t r = (int64_t)(blockIdx.x / strips) * kRows + threadIdx.x / kLanes;
    const int64_t b0 = (int64_t)(blockIdx.x % strips) * kSteps;
    const int lane = threadIdx.x % kLanes;
    if (r >= a.rows) return;
    const T *row = (const T *)a.x + r * a.ldx;
    float f[kSteps][kEach];
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
        if (b0 + i < a.col_blocks) load8<T, kAligned>(row, (b0 + i) * kBlock + lane * kEach, a.cols, f[i]);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (b0 + i >= a.col_blocks) break;
        const Steps s = steps_of(max_lanes<kLanes>(most8(f[i])));
        const int64_t c = (b0 + i) * kBlock + lane * kEach;
        store8<T>((char *)a.q + r * a.ldq, c, a.padded, (int)min(a.cols - c, (int64_t)kEach), f[i], s);
        if (lane == 0) a.scales[(b0 + i) * a.lds + r] = s.scale;
    }
}

template <typename T, bool kAligned>
__global__ __launch_bounds__(kThreads) void eb_quantize_blocks(QuantizeArgs a)
{
    constexpr int kParts = kBlock / kRows;
    __shared__ int most_of[kThreads / kWave];
    const int64_t block = blockIdx.x;
    const int64_t cb = block % a.col_blocks, rb = block / a.col_blocks % a.row_blocks, m = block / a.col_blocks / a.row_blocks;
    const int lane = threadIdx.x % kLanes;
    const int64_t c = cb * kBlock + lane * kEach;
    float f[kParts][kEach];
    int most = 0;
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        const int64_t r = rb * kBlock + i * kRows + threadIdx.x / kLanes;
        if (r < a.rows) {
            load8<T, kAligned>((const T *)a.x + (m * a.rows + r) * a.ldx, c, a.cols, f[i]);
            most = max(most, most8(f[i]));
        }
    }
    most = max_lanes<kWave>(most);
    if (threadIdx.x % kWave == 0) most_of[threadIdx.x / kWave] = most;
    __syncthreads();
    most = max(max(most_of[0], most_of[1]), max(most_of[2], most_of[3]));
    const Steps s = steps_of(most);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        const int64_t r = rb * kBlock + i * kRows + threadIdx.x / kLanes;
        if (r >= a.rows) continue;
        store8<T>((char *)a.q + (m * a.rows + r) * a.ldq, c, a.padded, (int)min(a.cols - c, (int64_t)kEach), f[i], s);
    }
    if (threadIdx.x == 0) a.scales[block] = s.scale;
}

template <typename T>
void *kernel_of(bool blocks, bool aligned)
{
    if (blocks) return aligned ? (void *)eb_quantize_blocks<T, true> : (void *)eb_quantize_blocks<T, false>;
    return aligned ? (void *)eb_quantize_rows<T, true> : (void *)eb_quantize_rows<T, false>;
}

int quantize_impl(const char *who, int32_t matrices, int64_t rows, int64_t cols, const void *x, int32_t dtype, int64_t ldx,
                  int32_t block_rows, void *q, int64_t ldq, float *scales, int64_t lds, void *stream)
{
    constexpr int64_t kMost = std::numeric_limits<int32_t>::max();
    if (matrices < 0 || rows < 0 || cols < 1) return fail(EB_ERR_INVALID, "%s: negative matrices or rows, or no columns", who);
    if (dtype != EB_F32 && dtype != EB_F16 && dtype != EB_BF16) return fail(EB_ERR_INVALID, "%s: unknown dtype", who);
    if (block_rows != 1 && block_rows != kBlock) return fail(EB_ERR_INVALID, "%s: block_rows must be 1 or 128", who);
    if (matrices == 0 || rows == 0) return EB_OK;
    if (!x || !q || !scales) return fail(EB_ERR_INVALID, "%s: NULL x, q or scales", who);
    if (ldx < cols || ldq < cols || ldq % 16 != 0 || (uintptr_t)q % 16 != 0)
        return fail(EB_ERR_INVALID, "%s: ldx or ldq below cols, or q or ldq not a multiple of 16 bytes", who);
    if (rows > kMost || matrices > std::numeric_limits<int64_t>::max() / 16 / rows / ldx || matrices > std::numeric_limits<int64_t>::max() / rows / ldq)
        return fail(EB_ERR_UNSUPPORTED, "%s: matrices too large", who);
    QuantizeArgs a{};
    a.x = x;
    a.q = q;
    a.scales = scales;
    a.ldx = ldx;
    a.ldq = ldq;
    a.lds = lds;
    a.cols = cols;
    a.padded = (cols + 15) / 16 * 16;
    a.col_blocks = (cols + kBlock - 1) / kBlock;
    const int es = dtype == EB_F32 ? 4 : 2;
    const bool aligned = (uintptr_t)x % 16 == 0 && ldx * es % 16 == 0;
    int64_t grid;
    if (block_rows == 1) {
        a.rows = matrices * rows;
        if (lds < a.rows || lds > std::numeric_limits<int64_t>::max() / 4 / a.col_blocks)
            return fail(EB_ERR_INVALID, "%s: lds below the rows, or too large", who);
        const int64_t strips = (a.col_blocks + kSteps - 1) / kSteps, lines = (a.rows + kRows - 1) / kRows;
        grid = strips > kMost / lines ? kMost + 1 : strips * lines;
    } else {
        a.rows = rows;
        a.row_blocks = (rows + kBlock - 1) / kBlock;
        grid = a.col_blocks > kMost / a.row_blocks / matrices ? kMost + 1 : matrices * a.row_blocks * a.col_blocks;
    }
    if (grid > std::numeric_limits<uint32_t>::max() / kThreads) // a launch's threads are counted in 32 bits
        return fail(EB_ERR_UNSUPPORTED, "%s: more blocks than one launch holds", who);
    void *kernel = dtype == EB_F32 ? kernel_of<float>(block_rows != 1, aligned)
                   : dtype == EB_F16 ? kernel_of<_Float16>(block_rows != 1, aligned)
                                     : kernel_of<Bf16>(block_rows != 1, aligned);
    void *args[] = {&a};
    const hipError_t err = hipLaunchKernel(kernel, dim3((unsigned)grid), dim3(kThreads), args, 0, (hipStream_t)stream);
    return err == hipSuccess ? EB_OK : fail(EB_ERR_HIP, "%s: kernel launch failed: %s", who, hipGetErrorString(err));
}

} // namespace

extern "C" int eb_quantize_fp8(int32_t matrices, int64_t rows, int64_t cols, const void *x, int32_t dtype, int64_t ldx,
                               int32_t block_rows, void *q, int64_t ldq, float *scales, int64_t lds, void *stream)
{
    try {
        return quantize_impl("eb_quantize_fp8", matrices, rows, cols, x, dtype, ldx, block_rows, q, ldq, scales, lds, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_quantize_fp8");
    }
}
