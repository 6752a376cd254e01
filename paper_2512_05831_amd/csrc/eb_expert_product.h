// What the kernels of eb_expert_product share: their arguments, the tile of an
// expert's slots that a workgroup takes, K's last block, and the epilogue.
//
// All of them multiply 16 weight rows by 16 tokens, the weights as the matrix
// instruction's first operand: lane l holds row l % 16 of both operands (a
// weight row, a token) and 32 of a block's 128 bytes of k, its chunks l / 16 and
// l / 16 + 4 of 16 bytes (any order of k serves as long as both operands have
// the same), and of the result token l % 16 and the weight rows
// l / 16 * 4 + 0 .. 3.  So the factor of a token's scale is one register per 16
// tokens, and a lane's results are four neighbouring outputs of one token.
//
// A product over one block of 128 starts from zero and is added to the fp32
// sum under x_scale * w_scale: four multiply-adds per 16 x 16, which the vector
// unit does while the matrix unit is at the next ones.
//
// The 8-bit matrix unit adds the products of eight neighbouring k with the bits
// cut that lie more than 13 below the largest of the eight: measured 1.5e-5 of
// the root mean square of sums of 128 normal values, with either instruction
// (16x16x128, 16x16x32), and in general less than 2^-10 of the largest of each
// eight.  The 16-bit unit is exact to fp32 on the same values, widened (9e-9), at
// half the rate.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include <type_traits>

#include "../../include/eb.h"
#include "../../include/eb_experts.h"
#include "eb_experts.h"

namespace eb_product {

using namespace eb_experts;

struct ProductArgs {
    const char *x, *w;
    const float *x_scales, *w_scales, *bias;
    const int32_t *tokens, *offsets;
    void *out;
    float *out_scales;
    int64_t ldx, ldxs, ldw, ldo, ldos;
    int64_t x_rows;
    int32_t M, E, N, K;
    int32_t width;       // output columns: N, or N / 2 under a gate
    int32_t k_blocks;    // ceil(K / 128)
    int32_t row_blocks;  // ceil(width / 128): blocks of weight rows, of one half under a gate
    int32_t w_blocks;    // of a whole expert
    int32_t relu;
    int32_t out_type;
    int32_t vector_out;  // rows of out start at multiples of 16 bytes
    int32_t column_tiles;
};

// A workgroup's slots: [first, end) of expert e's, at most the tile's height.
struct SlotTile {
    int32_t expert, first, end;
};

// The index-th tile of kHeight slots, counted over the experts' slots in order;
// expert -1 past the last.  Every wave finds it for itself, 64 experts at a
// time.
template <int kHeight>
__device__ __forceinline__ SlotTile slot_tile(const ProductArgs &a, int32_t index)
{
    if (!a.offsets) {
        const int64_t first = (int64_t)index * kHeight;
        if (first >= a.M) return {-1, 0, 0};
        return {0, (int32_t)first, (int32_t)min((int64_t)a.M, first + kHeight)};
    }
    const int lane = threadIdx.x % kWave;
    for (int32_t e0 = 0; e0 < a.E; e0 += kWave) {
        const int32_t e = e0 + lane;
        int32_t lo = 0, hi = 0;
        if (e < a.E) {
            lo = min(max(a.offsets[e], 0), a.M);
            hi = min(max(a.offsets[e + 1], lo), a.M);
        }
        const int32_t n = (int32_t)(((int64_t)hi - lo + kHeight - 1) / kHeight);
        int32_t upto = n;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int32_t o = __shfl_up(upto, d);
            upto += lane >= d ? o : 0;
        }
        const uint64_t past = __ballot(upto > index);
        if (past) {
            const int at = __ffsll((long long)past) - 1;
            const int32_t first = lo + (index - (upto - n)) * kHeight;
            const int32_t from = __shfl(first, at), to = __shfl(hi, at);
            return {__builtin_amdgcn_readfirstlane(e0 + at), __builtin_amdgcn_readfirstlane(from),
                    __builtin_amdgcn_readfirstlane(from + min(to - from, kHeight))};
        }
        index -= __shfl(upto, kWave - 1);
    }
    return {-1, 0, 0};
}

// The first n bytes of 16 (any n), zeros behind.
__device__ __forceinline__ i32x4 first_bytes(i32x4 v, int n)
{
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int m = n - 4 * d;
        v[d] = m >= 4 ? v[d] : m <= 0 ? 0 : v[d] & ((1 << 8 * m) - 1);
    }
    return v;
}

// The operand of a matrix instruction from its two chunks.
__device__ __forceinline__ i32x8 operand(i32x4 lo, i32x4 hi)
{
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Four times eight e4m3 values as bf16 (exact): the operands of the four matrix
// instructions over 32 that make up a block.
struct Wide {
    bf16x8 part[4];
};

__device__ __forceinline__ Wide widen8(i32x8 v)
{
    Wide o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i], 1.f, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i], 1.f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i + 1], 1.f, false);
        const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * i + 1], 1.f, true);
        o.part[i] = bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    return o;
}

// 16 weight rows times 16 tokens over a block of 128, in the 16-bit unit.
__device__ __forceinline__ f32x4 block_product(const Wide &w, const Wide &x)
{
    f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.part[i], x.part[i], p, 0, 0, 0);
    return p;
}

// The same in the 8-bit unit.
__device__ __forceinline__ f32x4 block_product(i32x8 w, i32x8 x)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}

// Four values rounded to nearest even in 16 bits.
template <typename T>
__device__ __forceinline__ uint2 pack16(f32x4 v)
{
    typedef T pair __attribute__((ext_vector_type(2)));
    return make_uint2(__builtin_bit_cast(uint32_t, pair{(T)v[0], (T)v[1]}), __builtin_bit_cast(uint32_t, pair{(T)v[2], (T)v[3]}));
}

// Four outputs of a slot from `column`, as bits of kSize bytes each.
template <int kSize, typename Bits>
__device__ __forceinline__ void store4(const ProductArgs &a, int64_t slot, int32_t column, Bits bits)
{
    static_assert(sizeof(Bits) == 4 * kSize, "four outputs");
    using Element = std::conditional_t<kSize == 4, uint32_t, std::conditional_t<kSize == 2, uint16_t, uint8_t>>;
    Element *p = (Element *)a.out + slot * a.ldo + column;
    if (a.vector_out && column + 4 <= a.width) {
        *(Bits *)p = bits;
    } else {
        Element e[4];
        __builtin_memcpy(e, &bits, sizeof e);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (column + i < a.width) p[i] = e[i];
    }
}

__device__ __forceinline__ f32x4 bias4(const float *bias, int32_t row, int32_t end)
{
    f32x4 b;
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = bias[min(row + i, end - 1)]; // any past the end: they are not stored
    return b;
}

// g / (1 + exp(-g)).  The hardware's 2^x and reciprocal are within an ulp, and
// the exponent's rounding adds |g| ulps to exp(-g): a few ulps where it counts
// beside the 1, and far less than an ulp of g of what is left for large -g.
__device__ __forceinline__ float silu(float g)
{
    return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269502f));
}

// The sums of kRows x kTokens tiles (weight rows of one wave) to outputs: bias,
// activation; under a gate rows [0, kRows / 2) of the tiles are the gate's and
// the others the outputs they gate.  Returns the output tiles in `s`.
template <int kRows, int kTokens, bool kGate>
__device__ __forceinline__ void finish(const ProductArgs &a, int32_t expert, int32_t column, f32x4 (&s)[kRows][kTokens])
{
    constexpr int kOut = kGate ? kRows / 2 : kRows;
    const int part = threadIdx.x % kWave / 16 * 4;
    if (a.bias) {
        const float *bias = a.bias + (int64_t)expert * a.N;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const bool up = kGate && r >= kOut;
            const f32x4 b = bias4(up ? bias + a.width : bias, column + (up ? r - kOut : r) * 16 + part, a.width);
#pragma unroll
            for (int t = 0; t < kTokens; ++t) s[r][t] += b;
        }
    }
    if constexpr (kGate) {
#pragma unroll
        for (int r = 0; r < kOut; ++r)
#pragma unroll
            for (int t = 0; t < kTokens; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[r][t][i] = silu(s[r][t][i]) * s[kOut + r][t][i];
    } else if (a.relu) {
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int t = 0; t < kTokens; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[r][t][i] = s[r][t][i] < 0.f ? 0.f : s[r][t][i]; // a NaN stays one
    }
}

// Floating-point outputs of one wave.  slot[t]: this lane's slot of token tile
// t, -1 where it is not to be written.
template <int kOut, int kRows, int kTokens>
__device__ __forceinline__ void store_floats(const ProductArgs &a, int32_t column, const int32_t (&slot)[kTokens],
                                             const f32x4 (&s)[kRows][kTokens])
{
    const int part = threadIdx.x % kWave / 16 * 4;
    auto store = [&](auto size, auto bits) {
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
            if (slot[t] < 0) continue;
#pragma unroll
            for (int r = 0; r < kOut; ++r) store4<decltype(size)::value>(a, slot[t], column + r * 16 + part, bits(s[r][t]));
        }
    };
    using Four = std::integral_constant<int, 4>;
    using Two = std::integral_constant<int, 2>;
    if (a.out_type == EB_F32) store(Four(), [](f32x4 v) { return v; });
    else if (a.out_type == EB_F16) store(Two(), [](f32x4 v) { return pack16<_Float16>(v); });
    else store(Two(), [](f32x4 v) { return pack16<__bf16>(v); });
}

// The largest magnitude of this wave's outputs for each of its tokens into
// `most` (LDS, one word per token of the workgroup's tile and output block,
// zero before).
template <int kOut, int kRows, int kTokens>
__device__ __forceinline__ void most_of_outputs(const f32x4 (&s)[kRows][kTokens], int *most)
{
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
        int m = 0;
#pragma unroll
        for (int r = 0; r < kOut; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) m = max(m, magnitude(s[r][t][i]));
        auto p = __builtin_amdgcn_permlane16_swap((unsigned)m, (unsigned)m, false, false);
        m = max((int)p[0], (int)p[1]);
        auto q = __builtin_amdgcn_permlane32_swap((unsigned)m, (unsigned)m, false, false);
        m = max((int)q[0], (int)q[1]);
        if (threadIdx.x % kWave < 16) atomicMax(&most[t * 16 + threadIdx.x % 16], m);
    }
}

// Four outputs in 8 bits under a scale.
__device__ __forceinline__ int pack_fp8(f32x4 v, float scale)
{
    const float f = 1.f / scale; // a product with it: within an ulp of the quotient
    return eb_experts::pack_fp8(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
}

// 8-bit outputs of one wave, once `most` is complete; `scales`: whether this
// wave writes the block's scales.
template <int kOut, int kRows, int kTokens>
__device__ __forceinline__ void store_fp8(const ProductArgs &a, int32_t column, const int32_t (&slot)[kTokens],
                                          const f32x4 (&s)[kRows][kTokens], const int *most, bool scales)
{
    const int lane = threadIdx.x % kWave, part = lane / 16 * 4;
#pragma unroll
    for (int t = 0; t < kTokens; ++t) {
        if (slot[t] < 0) continue;
        const float f = block_scale(most[t * 16 + lane % 16]);
#pragma unroll
        for (int r = 0; r < kOut; ++r) store4<1>(a, slot[t], column + r * 16 + part, pack_fp8(s[r][t], f));
        if (scales && lane < 16) a.out_scales[(int64_t)(column / kBlock) * a.ldos + slot[t]] = f;
    }
}

using KernelFn = void (*)(ProductArgs);

struct KernelPlan {
    KernelFn kernel;
    int32_t height;  // slots of a workgroup
    int32_t columns; // outputs of a workgroup
    int32_t threads;
    int32_t band;    // the grid holds a multiple of so many slot tiles
};

// Slots and weight rows of a workgroup: 256 x 256, 128 x 256, 64 x 128, 32 x 128.
enum class TileSize { kHuge, kLarge, kMedium, kSmall };

KernelPlan stream_kernel(bool gate, bool fp8);
KernelPlan tile_kernel(bool gate, bool fp8, bool wide, TileSize size);

} // namespace eb_product
