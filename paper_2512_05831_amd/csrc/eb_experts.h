// Shared by the experts' sources (eb_route_experts.hip, eb_quantize_fp8.hip,
// eb_expert_product*.hip); not part of the C ABI.
#pragma once

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <stdint.h>

namespace eb_experts {

constexpr int kWave = 64;
constexpr int kBlock = 128;              // values that share a scale
constexpr float kMostFp8 = 448.f;        // the largest e4m3 value
constexpr float kLeastScale = 0x1p-126f; // the smallest normal fp32

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct Bf16 {
    uint16_t bits;
};

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(_Float16 v) { return (float)v; }
__device__ __forceinline__ float widen(Bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }

// A row of 16 lanes rotated by S (a data-parallel primitive move, no LDS).
template <int S>
__device__ __forceinline__ int rotate16(int v)
{
    return __builtin_amdgcn_update_dpp(v, v, 0x120 + S, 0xF, 0xF, false);
}

// op over the L = 16 or 64 lanes of a group, the result in every lane.  `op`
// has to be commutative and associative, or its order a fixed tree (sums).
template <int L, typename Op>
__device__ __forceinline__ int reduce_lanes(int v, Op op)
{
    static_assert(L == 16 || L == 64, "a row of lanes, or a wave");
    v = op(v, rotate16<8>(v));
    v = op(v, rotate16<4>(v));
    v = op(v, rotate16<2>(v));
    v = op(v, rotate16<1>(v));
    if constexpr (L == 64) {
        auto a = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
        v = op((int)a[0], (int)a[1]);
        auto b = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
        v = op((int)b[0], (int)b[1]);
    }
    return v;
}

template <int L>
__device__ __forceinline__ int max_lanes(int v)
{
    return reduce_lanes<L>(v, [](int a, int b) { return a > b ? a : b; });
}

template <int L>
__device__ __forceinline__ int min_lanes(int v)
{
    return reduce_lanes<L>(v, [](int a, int b) { return a < b ? a : b; });
}

template <int L>
__device__ __forceinline__ int or_lanes(int v)
{
    return reduce_lanes<L>(v, [](int a, int b) { return a | b; });
}

template <int L>
__device__ __forceinline__ float sum_lanes(float v)
{
    return __int_as_float(
        reduce_lanes<L>(__float_as_int(v), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}

// LDS written by some lanes of a wave, then read by others of the same wave.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The bits of |v|: they order as the magnitudes do, with infinity and the NaNs
// (0x7F800000 and up) above every finite one.
__device__ __forceinline__ int magnitude(float v) { return __float_as_int(v) & 0x7FFFFFFF; }

// The scale of a block whose largest magnitude has these bits.
__device__ __forceinline__ float block_scale(int most)
{
    if (most >= 0x7F800000) return __int_as_float(0x7FC00000);
    const float s = __int_as_float(most) / kMostFp8;
    return s > kLeastScale ? s : kLeastScale;
}

// Four values to e4m3, rounded to nearest even, the first in the low byte.
__device__ __forceinline__ int pack_fp8(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

} // namespace eb_experts
