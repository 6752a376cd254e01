// The experts' activation, of values that wait in 8 bits or in floating point, and
// its gradient (include/eb_train.h): eb_activation, eb_activation_backward.
//
//   relu: h = max(v, 0), dv = dh where v > 0
//   gate: h = g p u, dg = dh u p (1 + g (1 - p)), du = dh g p, p = 1 / (1 + e^-g)
//
// Element by element but for the scales: bound by memory.  Eight neighbours a lane,
// 16 lanes a block of 128 that shares a scale; a workgroup takes 16 rows and up to
// kSteps blocks along them, so that scales that are neighbours in memory are read and
// written together.  32768 x 1024, gated, 8 bits in and out 28 us (3.7 TB/s);
// ReLU's gradient 24, 16-bit gated gradients 62 (5.4 TB/s).

#include <type_traits>

#include "eb_train.h"

namespace {

using namespace eb_train;

constexpr int kThreads = 256;
constexpr int kRows = kThreads / kLanes; // rows of a workgroup
constexpr int kSteps = 2;                // block columns of a workgroup

struct ActArgs {
    const void *v, *dh;
    Scales v_scales;
    Out out;
    int64_t rows, cols, ldv, lddh;
    int64_t width;  // of v: cols, or under a gate twice that
    int64_t blocks; // block columns that the workgroups walk
    bool gate;
};

// p = 1 / (1 + exp(-g)): the exponential with the rounding of its argument put right, by
// a factor c.  From g = 87 on p is 1.  Below -88.7 the exponential is infinite and p, as
// g p then, a zero of either sign (c means little there, but is neither 0 nor NaN; for
// -infinity it is NaN, and so is p).  A p below 2^-126 may be 0.
__device__ __forceinline__ float sigmoid(float g)
{
    constexpr float kLog2e = 1.44269502f, kRest = 1.92596303e-8f; // together log2(e) to 2^-50
    g = fminf(g, 87.f); // NaN: 87, whose p leaves the NaN of g p
    const float h = g * -kLog2e, l = fmaf(g, -kRest, fmaf(g, -kLog2e, -h));
    const float e = __builtin_amdgcn_exp2f(h), c = fmaf(l, 0.693147182f, 1.f);
    return __builtin_amdgcn_rcpf(fmaf(e, c, 1.f));
}

// Columns c .. c + 7 of v that lie in [lo, hi), to be settled where they are used.
template <bool kRagged, typename T>
__device__ __forceinline__ Raw<T> load_v(const ActArgs &a, int64_t row, int c, int lo, int hi)
{
    return fetch_raw<kRagged>((const T *)a.v + row * a.ldv + lo, c - lo, hi - lo);
}

// The scales of those, and their values.
template <bool kAcross, typename T>
__device__ __forceinline__ TwoScales scales_v(const ActArgs &a, int64_t row, int c, int hi)
{
    if constexpr (sizeof(T) == 1) return load_scales<kAcross>(a.v_scales, row, c, hi);
    else return {};
}

// (c and cols within the part.)
template <bool kRagged, bool kAcross, bool kBelow = false, typename T>
__device__ __forceinline__ void widen_v(const Raw<T> &r, const TwoScales &t, int c, int cols, float *f)
{
    widen8(settle_raw<kRagged, kBelow>(r, c, cols), f);
    if constexpr (sizeof(T) == 1) scale8<kAcross>(f, t);
}

template <typename T, bool kRagged>
__global__ __launch_bounds__(kThreads) void eb_activate(ActArgs a)
{
    const uint32_t strips = (a.blocks + kSteps - 1) / kSteps;
    const int64_t row = (int64_t)(blockIdx.x / strips) * kRows + threadIdx.x / kLanes;
    const int b0 = blockIdx.x % strips * kSteps, cols = (int)a.cols, width = (int)a.width;
    if (row >= a.rows) return;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int c = (b0 + s) * kBlock + threadIdx.x % kLanes * kEach;
        if (b0 + s >= a.blocks) return;
        float g[kEach], h[kEach];
        const Raw<T> first = load_v<kRagged, T>(a, row, c, 0, cols);
        const TwoScales of_g = scales_v<false, T>(a, row, c, cols);
        if (a.gate) {
            const Raw<T> second = load_v<kRagged, T>(a, row, cols + c, cols, width);
            const TwoScales of_u = scales_v<kRagged, T>(a, row, cols + c, width);
            float u[kEach];
            widen_v<kRagged, false>(first, of_g, c, cols, g);
            widen_v<kRagged, kRagged>(second, of_u, c, cols, u);
#pragma unroll
            for (int i = 0; i < kEach; ++i) h[i] = g[i] * sigmoid(g[i]) * u[i];
        } else {
            widen_v<kRagged, false>(first, of_g, c, cols, g);
#pragma unroll
            for (int i = 0; i < kEach; ++i) h[i] = g[i] > 0.f ? g[i] : g[i] == g[i] ? 0.f : g[i];
        }
        store_out<kRagged>(a.out, row, c, cols, h);
    }
}

// dg and du.
__device__ __forceinline__ float2 d_gate(float dh, float g, float u)
{
    const float p = sigmoid(g), dp = dh * p;
    return {dp * u * fmaf(g, 1.f - p, 1.f), dp * g};
}

// dg and du by the lane that has both g and u: floating-point outputs, and 8-bit
// ones whose blocks do not lie across the border between dg and du.
template <typename D, typename T, bool kRagged>
__global__ __launch_bounds__(kThreads) void eb_activate_back(ActArgs a)
{
    const uint32_t strips = (a.blocks + kSteps - 1) / kSteps;
    const int64_t row = (int64_t)(blockIdx.x / strips) * kRows + threadIdx.x / kLanes;
    const int b0 = blockIdx.x % strips * kSteps, cols = (int)a.cols, width = (int)a.width;
    if (row >= a.rows) return;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int c = (b0 + s) * kBlock + threadIdx.x % kLanes * kEach;
        if (b0 + s >= a.blocks) return;
        float dh[kEach], g[kEach], d[kEach];
        const Raw<D> of_h = fetch_raw<kRagged>((const D *)a.dh + row * a.lddh, c, cols);
        const Raw<T> first = load_v<kRagged, T>(a, row, c, 0, cols);
        const TwoScales scales_g = scales_v<false, T>(a, row, c, cols);
        if (!a.gate) {
            widen8(settle_raw<kRagged>(of_h, c, cols), dh);
            widen_v<kRagged, false>(first, scales_g, c, cols, g);
#pragma unroll
            for (int i = 0; i < kEach; ++i) d[i] = g[i] > 0.f ? dh[i] : 0.f;
            store_out<kRagged>(a.out, row, c, cols, d);
            continue;
        }
        const Raw<T> second = load_v<kRagged, T>(a, row, cols + c, cols, width);
        const TwoScales scales_u = scales_v<kRagged, T>(a, row, cols + c, width);
        float u[kEach], e[kEach];
        widen8(settle_raw<kRagged>(of_h, c, cols), dh);
        widen_v<kRagged, false>(first, scales_g, c, cols, g);
        const bool fp8 = a.out.type == EB_FP8; // whole blocks
        widen_v<kRagged, kRagged>(second, scales_u, c, cols, u);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const float2 v = d_gate(dh[i], g[i], u[i]);
            d[i] = v.x;
            e[i] = v.y;
        }
        Out of_u = a.out;
        if (!fp8) {
            of_u.p = (char *)a.out.p + cols * (int64_t)(a.out.type == EB_F32 ? 4 : 2);
            store8_of<kRagged>(a.out, row, c, cols, d);
            store8_of<kRagged>(of_u, row, c, cols, e);
            continue;
        }
        of_u.p = (char *)a.out.p + cols;
        of_u.scales = a.out.scales + cols / kBlock * a.out.lds;
        store_out<kRagged>(a.out, row, c, cols, d);
        store_out<kRagged>(of_u, row, c, cols, e);
    }
}

// The same from 8 bits to 8 bits, gated, columns a multiple of 128: bound by the vector
// unit as much as by memory (65536 x 1024 from bf16 dh: 87 us of GPU time, at a copy's rate 78; 102 before), so
// nothing is made twice: a block's place is the workgroup's, and u's scale is left to
// dg's, whose block is u's.
template <typename D>
__global__ __launch_bounds__(kThreads) void eb_activate_back_blocks(ActArgs a)
{
    const uint32_t strips = (a.blocks + kSteps - 1) / kSteps;
    const int64_t row = (int64_t)(blockIdx.x / strips) * kRows + threadIdx.x / kLanes;
    const int b0 = blockIdx.x % strips * kSteps, cols = (int)a.cols, blocks = (int)a.blocks;
    if (row >= a.rows) return;
    const int at = threadIdx.x % kLanes * kEach;
    const D *dh_row = (const D *)a.dh + row * a.lddh + at;
    const Fp8 *v_row = (const Fp8 *)a.v + row * a.ldv + at;
    char *out_row = (char *)a.out.p + row * a.out.ld + at;
    Raw<D> of_h[kSteps];
    Raw<Fp8> of_g[kSteps], of_u[kSteps];
    float sg[kSteps], su[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) { // a step past the last block takes that again, and writes it again
        const int b = min(b0 + s, blocks - 1), c = b * kBlock;
        of_h[s] = load_raw<false>(dh_row + c, 0, kEach);
        of_g[s] = load_raw<false>(v_row + c, 0, kEach);
        of_u[s] = load_raw<false>(v_row + cols + c, 0, kEach);
        sg[s] = (a.v_scales.p + (int64_t)b * a.v_scales.ld)[row];
        su[s] = (a.v_scales.p + (int64_t)(blocks + b) * a.v_scales.ld)[row];
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int b = min(b0 + s, blocks - 1), c = b * kBlock;
        float d[kEach], e[kEach], g[kEach], u[kEach];
        widen8(of_h[s], d);
        widen8(of_g[s], g);
        widen8(of_u[s], u);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const float2 v = d_gate(d[i], g[i] * sg[s], u[i]);
            d[i] = v.x;
            e[i] = v.y;
        }
        const int most_e = most_of_block(most8(e));
        const int most_d = most_of_block(most8(d));
        int scaled = magnitude(__int_as_float(most_d) * su[s]);
        Factor of_d = to_fp8(most_d);
        // Beyond fp32's range before u's scale it may be finite with it, and below the floor of
        // what a factor is made of it may lie above that: made again of the scaled u.
        if (most_d >= 0x7F800000 || (most_d != 0 && __int_as_float(most_d) <= kMostFp8 * kLeastScale)) {
            float dh[kEach];
            widen8(of_h[s], dh);
            widen8(of_g[s], g);
            widen8(of_u[s], u);
#pragma unroll
            for (int i = 0; i < kEach; ++i) d[i] = d_gate(dh[i], g[i] * sg[s], u[i] * su[s]).x;
            scaled = most_of_block(most8(d));
            of_d = to_fp8(scaled);
        } else if (__int_as_float(scaled) <= kMostFp8 * kLeastScale) { // the least scale: the values count
#pragma unroll
            for (int i = 0; i < kEach; ++i) d[i] *= su[s];
            of_d = kToLeast;
        }
        *(int2 *)(out_row + c) = eight_bits<false>(d, of_d, scaled >= 0x7F800000, kEach);
        *(int2 *)(out_row + cols + c) = eight_bits<false>(e, to_fp8(most_e), most_e >= 0x7F800000, kEach);
        if (threadIdx.x % kLanes == 0) {
            (a.out.scales + (int64_t)b * a.out.lds)[row] = scale_of(scaled);
            (a.out.scales + (int64_t)(blocks + b) * a.out.lds)[row] = scale_of(most_e);
        }
    }
}

// A lane of a block of dv, which may lie across the border, takes dg where its
// columns are g's, du where they are u's; dh and g are read for each. 32768 x 1016
// 75 us, 1023 columns 83 (1024, without a border inside a block, 41).
template <typename D, typename T, bool kRagged>
__global__ __launch_bounds__(kThreads) void eb_activate_back_across(ActArgs a)
{
    const uint32_t strips = (a.blocks + kSteps - 1) / kSteps;
    const int64_t row = (int64_t)(blockIdx.x / strips) * kRows + threadIdx.x / kLanes;
    const int b0 = blockIdx.x % strips * kSteps, cols = (int)a.cols, width = (int)a.width;
    if (row >= a.rows) return;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int at = (b0 + s) * kBlock + threadIdx.x % kLanes * kEach;
        if (b0 + s >= a.blocks) return;
        float d[kEach] = {};
        // Columns c on of dg, or of du; those outside [0, cols) are another's, or padding.
        auto take = [&](int c, bool first, auto aligned) {
            constexpr bool kAcross = kRagged && !decltype(aligned)::value;
            const Raw<D> of_h = fetch_raw<kRagged>((const D *)a.dh + row * a.lddh, c, cols);
            const Raw<T> of_g = load_v<kRagged, T>(a, row, c, 0, cols), of_u = load_v<kRagged, T>(a, row, cols + c, cols, width);
            const TwoScales scales_g = scales_v<kAcross, T>(a, row, c, cols), scales_u = scales_v<kRagged, T>(a, row, cols + c, width);
            float dh[kEach], g[kEach], u[kEach];
            widen8(settle_raw<kRagged, kAcross>(of_h, c, cols), dh);
            widen_v<kRagged, kAcross, kAcross>(of_g, scales_g, c, cols, g);
            widen_v<kRagged, kRagged, kAcross>(of_u, scales_u, c, cols, u);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const float2 v = d_gate(dh[i], g[i], u[i]);
                const float one = first ? v.x : v.y;
                if (!kRagged) d[i] = one; // of columns past the last zero
                else if (c + i >= 0 && c + i < cols) d[i] = one;
            }
        };
        if constexpr (!kRagged) {
            take(at < cols ? at : at - cols, at < cols, std::true_type());
        } else {
            if (at < cols) take(at, true, std::true_type());
            if (at + kEach > cols) take(at - cols, false, std::false_type()); // both, where the border lies within
        }
        store_out<kRagged>(a.out, row, at, width, d);
    }
}

int check(const char *who, int64_t rows, int64_t cols, int32_t act, int32_t v_type, int32_t out_type)
{
    if (rows < 0 || cols < 1) return fail(EB_ERR_INVALID, "%s: negative rows, or no columns", who);
    if (act != EB_ACT_RELU && act != EB_ACT_SILU_GATE) return fail(EB_ERR_INVALID, "%s: act must be EB_ACT_RELU or EB_ACT_SILU_GATE", who);
    if ((!floating(v_type) && v_type != EB_FP8) || (!floating(out_type) && out_type != EB_FP8))
        return fail(EB_ERR_INVALID, "%s: unknown v_type or out_type", who);
    if (cols > (int64_t)1 << 29) return fail(EB_ERR_UNSUPPORTED, "%s: more than 2^29 columns", who);
    return EB_OK;
}

int launch_rows(const char *who, void *kernel, ActArgs &a, void *stream)
{
    const int64_t strips = (a.blocks + kSteps - 1) / kSteps, lines = a.rows / kRows + (a.rows % kRows != 0);
    return launch(who, kernel, lines > kMax32 / strips ? kMax32 : lines * strips, kThreads, &a, stream);
}

template <typename T>
void *act_kernel(bool ragged)
{
    return ragged ? (void *)eb_activate<T, true> : (void *)eb_activate<T, false>;
}

int act_impl(const char *who, int64_t rows, int64_t cols, int32_t act, const void *v, int32_t v_type, int64_t ldv, const float *v_scales,
             int64_t ldvs, int32_t out_type, void *h, int64_t ldh, float *h_scales, int64_t ldhs, void *stream)
{
    if (int rc = check(who, rows, cols, act, v_type, out_type)) return rc;
    ActArgs a{};
    a.gate = act == EB_ACT_SILU_GATE;
    a.width = a.gate ? 2 * cols : cols;
    if (int rc = check_matrix(who, "v", v, v_type, rows, a.width, ldv, v_scales, ldvs)) return rc;
    if (int rc = check_matrix(who, "h", h, out_type, rows, cols, ldh, h_scales, ldhs)) return rc;
    if (rows == 0) return EB_OK;
    a.v = v;
    a.v_scales = {v_scales, ldvs};
    a.out = {h, h_scales, ldh, ldhs, out_type};
    a.rows = rows;
    a.cols = cols;
    a.ldv = ldv;
    a.blocks = (cols + kBlock - 1) / kBlock;
    const bool ragged = cols % kEach != 0;
    void *kernel = v_type == EB_F32   ? act_kernel<float>(ragged)
                   : v_type == EB_F16 ? act_kernel<_Float16>(ragged)
                   : v_type == EB_FP8 ? act_kernel<Fp8>(ragged)
                                      : act_kernel<Bf16>(ragged);
    return launch_rows(who, kernel, a, stream);
}

template <typename D, typename T>
void *back_kernel(bool across, bool ragged)
{
    if (across) return ragged ? (void *)eb_activate_back_across<D, T, true> : (void *)eb_activate_back_across<D, T, false>;
    return ragged ? (void *)eb_activate_back<D, T, true> : (void *)eb_activate_back<D, T, false>;
}

template <typename D>
void *back_kernel(int32_t v_type, bool across, bool ragged)
{
    if (v_type == EB_F32) return back_kernel<D, float>(across, ragged);
    if (v_type == EB_F16) return back_kernel<D, _Float16>(across, ragged);
    if (v_type == EB_FP8) return back_kernel<D, Fp8>(across, ragged);
    return back_kernel<D, Bf16>(across, ragged);
}

int back_impl(const char *who, int64_t rows, int64_t cols, int32_t act, const void *dh, int32_t dh_type, int64_t lddh, const void *v,
              int32_t v_type, int64_t ldv, const float *v_scales, int64_t ldvs, int32_t out_type, void *dv, int64_t lddv, float *dv_scales,
              int64_t lddvs, void *stream)
{
    if (int rc = check(who, rows, cols, act, v_type, out_type)) return rc;
    if (!floating(dh_type)) return fail(EB_ERR_INVALID, "%s: unknown dh_type", who);
    ActArgs a{};
    a.gate = act == EB_ACT_SILU_GATE;
    a.width = a.gate ? 2 * cols : cols;
    if (int rc = check_matrix(who, "dh", dh, dh_type, rows, cols, lddh, nullptr, 0)) return rc;
    if (int rc = check_matrix(who, "v", v, v_type, rows, a.width, ldv, v_scales, ldvs)) return rc;
    if (int rc = check_matrix(who, "dv", dv, out_type, rows, a.width, lddv, dv_scales, lddvs)) return rc;
    if (rows == 0) return EB_OK;
    a.v = v;
    a.dh = dh;
    a.v_scales = {v_scales, ldvs};
    a.out = {dv, dv_scales, lddv, lddvs, out_type};
    a.rows = rows;
    a.cols = cols;
    a.ldv = ldv;
    a.lddh = lddh;
    const bool across = a.gate && out_type == EB_FP8 && cols % kBlock != 0;
    a.blocks = ((across ? a.width : cols) + kBlock - 1) / kBlock;
    if (a.gate && v_type == EB_FP8 && out_type == EB_FP8 && !across) {
        void *kernel = dh_type == EB_F32   ? (void *)eb_activate_back_blocks<float>
                       : dh_type == EB_F16 ? (void *)eb_activate_back_blocks<_Float16>
                                           : (void *)eb_activate_back_blocks<Bf16>;
        return launch_rows(who, kernel, a, stream);
    }
    void *kernel = dh_type == EB_F32   ? back_kernel<float>(v_type, across, cols % kEach != 0)
                   : dh_type == EB_F16 ? back_kernel<_Float16>(v_type, across, cols % kEach != 0)
                                       : back_kernel<Bf16>(v_type, across, cols % kEach != 0);
    return launch_rows(who, kernel, a, stream);
}

} // namespace

extern "C" int eb_activation(int64_t rows, int64_t cols, int32_t act, const void *v, int32_t v_type, int64_t ldv, const float *v_scales,
                             int64_t ldvs, int32_t out_type, void *h, int64_t ldh, float *h_scales, int64_t ldhs, void *stream)
{
    try {
        return act_impl("eb_activation", rows, cols, act, v, v_type, ldv, v_scales, ldvs, out_type, h, ldh, h_scales, ldhs, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_activation");
    }
}

extern "C" int eb_activation_backward(int64_t rows, int64_t cols, int32_t act, const void *dh, int32_t dh_type, int64_t lddh, const void *v,
                                      int32_t v_type, int64_t ldv, const float *v_scales, int64_t ldvs, int32_t out_type, void *dv,
                                      int64_t lddv, float *dv_scales, int64_t lddvs, void *stream)
{
    try {
        return back_impl("eb_activation_backward", rows, cols, act, dh, dh_type, lddh, v, v_type, ldv, v_scales, ldvs, out_type, dv, lddv,
                         dv_scales, lddvs, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_activation_backward");
    }
}
