// Shared by what trains a layer of experts (eb_layer_norm*.hip, eb_activation.hip,
// eb_sort_rows.hip, eb_weight_gradient*); not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <stddef.h>
#include <stdint.h>

#include <limits>
#include <type_traits>

#include "../../include/eb.h"
#include "../../include/eb_experts.h"
#include "../../include/eb_train.h"
#include "eb_experts.h"
#include "eb_internal.h"

namespace eb_train {

using namespace eb_experts;
using eb_detail::fail;

constexpr int kEach = 8;               // neighbouring values that a lane holds
constexpr int kLanes = kBlock / kEach; // lanes of a block that shares a scale
constexpr int64_t kMax64 = std::numeric_limits<int64_t>::max();
constexpr int64_t kMax32 = std::numeric_limits<int32_t>::max();

struct Fp8 {
    uint8_t bits;
};

// Accesses of any alignment: the hardware's, at their full width.
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef int i32x2_any __attribute__((ext_vector_type(2), aligned(1)));

// Eight neighbouring values as they lie in memory.
template <typename T>
struct Raw {
    T v[kEach];
};

// Eight values moved down by n >= 0 places (kUp: up), zeros in their place; 8 and
// more: all zeros.
template <bool kUp, typename T>
__device__ __forceinline__ Raw<T> moved(Raw<T> r, int n)
{
    if constexpr (sizeof(T) == 1) {
        uint64_t v;
        __builtin_memcpy(&v, &r, 8);
        v = n >= 8 ? 0 : kUp ? v << 8 * n : v >> 8 * n;
        __builtin_memcpy(&r, &v, 8);
    } else {
        constexpr int kWords = 2 * sizeof(T), kOne = (int)sizeof(T);
        uint32_t w[kWords];
        __builtin_memcpy(w, &r, sizeof(r));
        auto by = [&](int words, bool really) { // each word is read before it is written
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
                const int i = kUp ? kWords - 1 - j : j, from = kUp ? i - words : i + words;
                const uint32_t other = from >= 0 && from < kWords ? w[from] : 0;
                w[i] = really ? other : w[i];
            }
        };
        if constexpr (kOne == 4) {
            by(1, n & 1);
        } else {
            const uint32_t bits = n & 1 ? 16 : 0;
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
                const int i = kUp ? kWords - 1 - j : j, from = kUp ? i - 1 : i + 1;
                const uint32_t other = from >= 0 && from < kWords ? w[from] : 0;
                const uint64_t two = kUp ? (uint64_t)w[i] << 32 | other : (uint64_t)other << 32 | w[i];
                w[i] = kUp ? (uint32_t)((two << bits) >> 32) : (uint32_t)(two >> bits);
            }
        }
        by(kOne / 2, n & 2);
        by(kOne, n & 4);
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = n < 8 ? w[i] : 0;
        __builtin_memcpy(&r, w, sizeof(r));
    }
    return r;
}

template <typename T>
__device__ __forceinline__ Raw<T> load_whole(const T *at)
{
    Raw<T> r;
    if constexpr (sizeof(T) == 1) {
        const i32x2_any w = *(const i32x2_any *)at;
        __builtin_memcpy(&r, &w, 8);
    } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const i32x4_any w = *(const i32x4_any *)((const char *)at + 16 * i);
            __builtin_memcpy((char *)&r + 16 * i, &w, 16);
        }
    }
    return r;
}

// Those from column c of a row on, which has columns [0, cols); zeros outside.
// kRagged: cols may be any; with kBelow c too may be below 0; else both are multiples
// of 8.
// fetch_raw loads, settle_raw puts in place. Of a ragged row the chunk at an end is
// loaded whole too, from within the row, and moved where it is used: no branch on the
// data lies between the loads of several chunks, which then go out together. With
// branches instead: layer norm's gradients, 16384 x 3327 in bf16 by 8 bits, 122 us in
// place of 90; a gated activation's to 8 bits, 32768 x 1023, 130 in place of 83.
template <bool kRagged, typename T>
__device__ __forceinline__ Raw<T> fetch_raw(const T *row, int c, int cols)
{
    if constexpr (!kRagged) return load_whole(row + (c < cols ? c : 0));
    else if (cols >= kEach) return load_whole(row + max(0, min(c, cols - kEach)));
    using Bits = std::conditional_t<sizeof(T) == 1, uint8_t, std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>>;
    constexpr int kOf = 4 / (int)sizeof(T); // values of a word
    uint32_t w[kEach / kOf] = {};
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (c + i >= 0 && c + i < cols) w[i / kOf] |= (uint32_t)((const Bits *)row)[c + i] << i % kOf * 8 * (int)sizeof(T);
    Raw<T> r;
    __builtin_memcpy(&r, w, sizeof(r));
    return r;
}

template <bool kRagged, bool kBelow = false, typename T>
__device__ __forceinline__ Raw<T> settle_raw(Raw<T> r, int c, int cols)
{
    if constexpr (!kRagged) {
        int w[2 * sizeof(T)];
        __builtin_memcpy(w, &r, sizeof(r));
#pragma unroll
        for (int i = 0; i < (int)(2 * sizeof(T)); ++i) w[i] = c < cols ? w[i] : 0;
        __builtin_memcpy(&r, w, sizeof(r));
    } else if (cols >= kEach) {
        if (c > cols - kEach) r = moved<false>(r, c - (cols - kEach));
        if (kBelow && c < 0) r = moved<true>(r, -c);
    }
    return r;
}

template <bool kRagged, typename T>
__device__ __forceinline__ Raw<T> load_raw(const T *row, int c, int cols)
{
    return settle_raw<kRagged>(fetch_raw<kRagged>(row, c, cols), c, cols);
}

template <typename T>
__device__ __forceinline__ void widen8(const Raw<T> &r, float *f)
{
    if constexpr (sizeof(T) == 1) {
        int w[2];
        __builtin_memcpy(w, &r, 8);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
            f[4 * i + 0] = lo[0];
            f[4 * i + 1] = lo[1];
            f[4 * i + 2] = hi[0];
            f[4 * i + 3] = hi[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) f[i] = widen(r.v[i]);
    }
}

// The scales of an 8-bit matrix: that of row r's block b at b * ld + r.
struct Scales {
    const float *p;
    int64_t ld;
};

// The scales of columns c .. c + 7 of a row of an 8-bit matrix of `cols` columns: they
// lie in one block, or, where c is no multiple of 8 (kAcross), in two.
struct TwoScales {
    float first, second;
    int border; // values from this one on have the second
};

template <bool kAcross>
__device__ __forceinline__ TwoScales load_scales(const Scales &s, int64_t row, int c, int cols)
{
    const int lo = max(c, 0), hi = min(c + kEach, cols) - 1, b = lo / kBlock;
    const bool none = lo > hi; // zeros, whatever the scales
    TwoScales t;
    t.first = s.p[(none ? 0 : b) * s.ld + row];
    if (none) t.first = 0.f;
    if constexpr (kAcross) {
        t.second = s.p[(none ? 0 : hi / kBlock) * s.ld + row];
        if (none) t.second = 0.f;
        t.border = (b + 1) * kBlock - c;
    }
    return t;
}

template <bool kAcross>
__device__ __forceinline__ void scale8(float *f, const TwoScales &t)
{
#pragma unroll
    for (int i = 0; i < kEach; ++i) f[i] *= !kAcross || i < t.border ? t.first : t.second;
}

// The bits of the largest magnitude.
__device__ __forceinline__ int most8(const float *f)
{
    int m = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) m = max(m, magnitude(f[i]));
    return m;
}

// The largest over the 16 lanes of a block, all of them there, in every lane.
__device__ __forceinline__ int most_of_block(int v)
{
    v = max(v, __builtin_amdgcn_mov_dpp(v, 0x128, 0xF, 0xF, true)); // rotated by 8
    v = max(v, __builtin_amdgcn_mov_dpp(v, 0x124, 0xF, 0xF, true));
    v = max(v, __builtin_amdgcn_mov_dpp(v, 0x122, 0xF, 0xF, true));
    return max(v, __builtin_amdgcn_mov_dpp(v, 0x121, 0xF, 0xF, true));
}

// What brings a block's values to e4m3: 448 / largest, and what its rounding left.
struct Factor {
    float by, rest;
};

// Eight values times that as e4m3; NaNs where a block's scale is one. `left`: how many
// of them there are (the others are zeros).  The product is the quotient rounded once
// to fp32 (but for one in 2^20): values that lie in the middle of two e4m3 numbers
// stay there.
// kOnce false: rounded twice, where the values have roundings of their own behind them.
template <bool kOnce>
__device__ __forceinline__ int2 eight_bits(const float *f, Factor k, bool nan, int left)
{
    float p[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) p[i] = kOnce ? fmaf(f[i], k.by, f[i] * k.rest) : f[i] * k.by;
    int2 v;
    v.x = pack_fp8(p[0], p[1], p[2], p[3]);
    v.y = pack_fp8(p[4], p[5], p[6], p[7]);
    if (nan) {
        const uint64_t all = 0x7F7F7F7F7F7F7F7Full, some = left >= 8 ? all : left <= 0 ? 0 : all >> 8 * (8 - left);
        v.x = (int)some;
        v.y = (int)(some >> 32);
    }
    return v;
}

__device__ __forceinline__ uint32_t pack16(_Float16 a, _Float16 b)
{
    uint16_t x, y;
    __builtin_memcpy(&x, &a, 2);
    __builtin_memcpy(&y, &b, 2);
    return x | (uint32_t)y << 16;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    uint32_t w;
    __builtin_memcpy(&w, &v, 4);
    return w;
}

// Eight fp32 values to columns c .. c + 7 of a row in a floating-point type (a
// code of eb.h), each rounded once to nearest even; of the last chunk of a ragged row
// those past cols are left out.
template <bool kRagged>
__device__ __forceinline__ void store8(void *row, int type, int c, int cols, const float *f)
{
    if (type == EB_F32) {
        float *to = (float *)row + c;
        if (!kRagged || c + kEach <= cols) {
            const i32x4_any lo = {__float_as_int(f[0]), __float_as_int(f[1]), __float_as_int(f[2]), __float_as_int(f[3])};
            const i32x4_any hi = {__float_as_int(f[4]), __float_as_int(f[5]), __float_as_int(f[6]), __float_as_int(f[7])};
            *(i32x4_any *)to = lo;
            *(i32x4_any *)(to + 4) = hi;
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (c + i < cols) to[i] = f[i];
        }
        return;
    }
    uint32_t w[4];
    if (type == EB_F16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack16((_Float16)f[2 * i], (_Float16)f[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
    }
    uint16_t *to = (uint16_t *)row + c;
    if (!kRagged || c + kEach <= cols) {
        const i32x4_any v = {(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
        *(i32x4_any *)to = v;
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (c + i < cols) to[i] = (uint16_t)(w[i / 2] >> 16 * (i % 2));
    }
}

// A matrix that a kernel writes: floating point, or 8 bits with scales.
struct Out {
    void *p;
    float *scales;
    int64_t ld, lds;
    int32_t type;
};

// The scale of a block whose largest magnitude has these bits: its 448th, rounded once
// (the quotient by a product, then what that leaves of the dividend), 2^-126 and more.
__device__ __forceinline__ float scale_of(int most)
{
    constexpr float kPart = 1.f / kMostFp8;
    const float m = __int_as_float(most), q = m * kPart;
    const float s = fmaxf(fmaf(fmaf(-kMostFp8, q, m), kPart, q), kLeastScale);
    return most >= 0x7F800000 ? __int_as_float(0x7FC00000) : s;
}

// The factor of such a block (the reciprocal instruction's, and steps of Newton's method).
__device__ __forceinline__ Factor to_fp8(int most)
{
    const float m = fmaxf(__int_as_float(most), kMostFp8 * kLeastScale) * 0x1p-4f, r = __builtin_amdgcn_rcpf(m); // both normal
    const float by = fmaf(fmaf(-m, r, 1.f), r, r) * (kMostFp8 * 0x1p-4f);
    return {by, fmaf(-m, by, kMostFp8 * 0x1p-4f) * r};
}

constexpr Factor kToLeast = {1.f / kLeastScale, 0.f}; // under the least scale

// Columns c .. c + 7 of a row in 8 bits, the row padded to 16 bytes: values that are
// `by` to be multiplied with, under a scale for the largest magnitude `most` (bits).
template <bool kOnce = true>
__device__ __forceinline__ void store_fp8(const Out &o, int64_t row, int c, int cols, const float *f, Factor by, int most)
{
    if (c >= ((cols + 15) & ~15)) return;
    *(int2 *)((char *)o.p + row * o.ld + c) = eight_bits<kOnce>(f, by, most >= 0x7F800000, cols - c);
    if (c % kBlock == 0) o.scales[c / kBlock * o.lds + row] = scale_of(most);
}

// Columns c .. c + 7 of a row in floating point.
template <bool kRagged>
__device__ __forceinline__ void store8_of(const Out &o, int64_t row, int c, int cols, const float *f)
{
    if (c < cols) store8<kRagged>((char *)o.p + row * o.ld * (o.type == EB_F32 ? 4 : 2), o.type, c, cols, f);
}

// Columns c .. c + 7 of a row; in 8 bits the 16 lanes of a block call together.
template <bool kRagged>
__device__ __forceinline__ void store_out(const Out &o, int64_t row, int c, int cols, const float *f)
{
    if (o.type == EB_FP8) {
        const int most = most_of_block(most8(f));
        store_fp8(o, row, c, cols, f, to_fp8(most), most);
    } else {
        store8_of<kRagged>(o, row, c, cols, f);
    }
}

// Host side: checks shared by the entry points.

inline int element_bytes(int32_t type) { return type == EB_F32 ? 4 : type == EB_FP8 ? 1 : 2; }
inline bool floating(int32_t type) { return type == EB_F32 || type == EB_F16 || type == EB_BF16; }

// A matrix of rows x cols in `type`, its rows ld elements apart; an 8-bit one with
// its scales.
inline int check_matrix(const char *who, const char *what, const void *p, int32_t type, int64_t rows, int64_t cols,
                        int64_t ld, const float *scales, int64_t lds)
{
    const int es = element_bytes(type);
    if (rows == 0) return EB_OK;
    if (!p) return fail(EB_ERR_INVALID, "%s: %s is NULL", who, what);
    if (ld < cols) return fail(EB_ERR_INVALID, "%s: rows of %s overlap", who, what);
    if ((uintptr_t)p % es != 0) return fail(EB_ERR_INVALID, "%s: %s is not aligned to its elements", who, what);
    if (ld > kMax64 / 4 / rows) return fail(EB_ERR_UNSUPPORTED, "%s: %s exceeds 2^63 bytes", who, what);
    if (type != EB_FP8) return EB_OK;
    if ((uintptr_t)p % 16 != 0 || ld % 16 != 0)
        return fail(EB_ERR_INVALID, "%s: %s in 8 bits must be a multiple of 16 bytes, in its address and between rows", who, what);
    if (!scales || lds < rows) return fail(EB_ERR_INVALID, "%s: %s in 8 bits needs its scales, as many apart as it has rows", who, what);
    if (lds > kMax64 / 4 / ((cols + kBlock - 1) / kBlock)) return fail(EB_ERR_UNSUPPORTED, "%s: the scales of %s exceed 2^63 bytes", who, what);
    return EB_OK;
}

inline int launch(const char *who, void *kernel, int64_t grid, int threads, void *args, void *stream)
{
    // A launch's threads are counted in 32 bits.
    if (grid > std::numeric_limits<uint32_t>::max() / threads) return fail(EB_ERR_UNSUPPORTED, "%s: more work than one launch holds", who);
    void *list[] = {args};
    const hipError_t err = hipLaunchKernel(kernel, dim3((unsigned)grid), dim3((unsigned)threads), list, 0, (hipStream_t)stream);
    return err == hipSuccess ? EB_OK : fail(EB_ERR_HIP, "%s: kernel launch failed: %s", who, hipGetErrorString(err));
}

} // namespace eb_train
