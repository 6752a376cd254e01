// eb_weight_gradient (include/eb_train.h), its kernel: for every expert
//
//   dw[n, k] = sum over its slots m of dy[m, n] x[token of m, k]
//
// with the 16-bit matrix unit.  Both operands lie with the slots one below the other,
// while the unit wants eight slots of one column in a lane: a thread reads four
// columns of eight slots, turns them, and puts each column's eight 16-bit values into
// LDS as one piece of 16 bytes.
//   8-bit operands are widened on the way.  A slot's scales (of dy and of x, both one
// number for a tile of 128 x 128, whose edges are those of the scales' blocks) go into
// one operand as their product S, so that the other one, e4m3 or 16 bits, enters
// exactly.  The scaled one has up to 28 bits and takes several 16-bit parts where sums
// have to be exact, each multiplied with the other operand:
//   beside e4m3 or fp16, two parts in fp16, 22 bits.  Their range is short, so S is
//     divided by a power of two, kept above the largest S so far; where that grows
//     the sums are brought to the new one (exactly), and the outputs multiplied by the last;
//   beside bfloat16, three parts in that, 24 bits.
#pragma once

#include <type_traits>

#include "eb_train.h"

namespace eb_gradient {

using namespace eb_train;

constexpr int kThreads = 256;
constexpr int kTile = 128;  // columns of either operand
constexpr int kSlots = 64;  // of a step
constexpr int kChunks = kSlots / 8;
constexpr int kQuad = 4;    // columns of a thread
constexpr int kQuads = kTile / kQuad;

struct GradientArgs {
    const char *dy, *x;
    Scales dy_scales, x_scales;
    const int32_t *tokens, *offsets;
    void *dw;
    float *partial; // [splits][E][N, K], or NULL
    int64_t lddy, ldx, x_rows, lddw; // lddy, ldx in bytes
    int32_t M, E, N, K;
    int32_t n_tiles, k_tiles, splits;
    int32_t out_type;
    bool accumulate;
};

struct alignas(16) Piece { // eight slots of a column
    uint32_t w[4];
};

// How an operand of type T enters the matrix unit, in fp16 (kHalf) or bfloat16.
template <typename T, bool kScaled_, bool kHalf_, bool kExact>
struct Operand {
    using Type = T;
    static constexpr bool kScaled = kScaled_, kHalf = kHalf_;
    static constexpr bool kBits = !kScaled && std::is_same_v<T, std::conditional_t<kHalf, _Float16, Bf16>>; // as in memory
    static constexpr bool kSure = kBits || (std::is_same_v<T, Fp8> && !kScaled); // one 16-bit value holds it
    static constexpr int kParts = !kExact || kSure ? 1 : kHalf || !kScaled ? 2 : 3;
    static constexpr int kWords = sizeof(T); // 32-bit words of four values
};

// Four neighbouring columns of a slot.
template <typename T>
__device__ __forceinline__ void load_quad(const char *row, int c, int cols, uint32_t *w)
{
    constexpr int n = sizeof(T);
    typedef int i32_any __attribute__((aligned(1)));
    if (c + kQuad <= cols) {
        if constexpr (n == 1) {
            w[0] = *(const i32_any *)(row + c);
        } else {
            const i32x2_any v = *(const i32x2_any *)(row + (int64_t)c * n);
            w[0] = v.x;
            w[1] = v.y;
        }
    } else {
        T v[kQuad] = {};
#pragma unroll
        for (int i = 0; i < kQuad; ++i)
            if (c + i < cols) v[i] = ((const T *)row)[c + i];
        __builtin_memcpy(w, v, sizeof(v));
    }
}

template <typename T>
__device__ __forceinline__ void widen_quad(const uint32_t *w, float *f)
{
    if constexpr (std::is_same_v<T, Fp8>) {
        f[0] = __builtin_amdgcn_cvt_f32_fp8(w[0], 0);
        f[1] = __builtin_amdgcn_cvt_f32_fp8(w[0], 1);
        f[2] = __builtin_amdgcn_cvt_f32_fp8(w[0], 2);
        f[3] = __builtin_amdgcn_cvt_f32_fp8(w[0], 3);
    } else {
        T v[kQuad];
        __builtin_memcpy(v, w, sizeof(v));
#pragma unroll
        for (int i = 0; i < kQuad; ++i) f[i] = widen(v[i]);
    }
}

// Two values in 16 bits, and what that leaves of them.
template <bool kHalf>
__device__ __forceinline__ uint32_t pack_part(float &a, float &b)
{
    if constexpr (kHalf) {
        const _Float16 x = (_Float16)a, y = (_Float16)b;
        a -= (float)x;
        b -= (float)y;
        return pack16(x, y);
    } else {
        const uint32_t w = pack_bf16(a, b);
        a -= __uint_as_float(w << 16);
        b -= __uint_as_float(w & 0xFFFF0000u);
        return w;
    }
}

// The eight slots' four columns, turned: `to` is the first column's piece, the
// others kQuads pieces apart, the next parts kChunks * kTile.
template <typename O>
__device__ __forceinline__ void turn(const uint32_t (*raw)[O::kWords], const float *scale, Piece *to)
{
    Piece part[O::kParts][kQuad];
#pragma unroll
    for (int i = 0; i < 4; ++i) { // slots 2 i and 2 i + 1
        const uint32_t *a = raw[2 * i], *b = raw[2 * i + 1];
        if constexpr (O::kBits) {
#pragma unroll
            for (int j = 0; j < kQuad; ++j) part[0][j].w[i] = __builtin_amdgcn_perm(b[j / 2], a[j / 2], j % 2 ? 0x07060302 : 0x05040100);
        } else {
            float f[kQuad], g[kQuad];
            widen_quad<typename O::Type>(a, f);
            widen_quad<typename O::Type>(b, g);
#pragma unroll
            for (int j = 0; j < kQuad; ++j) {
                if constexpr (O::kScaled) {
                    f[j] *= scale[2 * i];
                    g[j] *= scale[2 * i + 1];
                }
#pragma unroll
                for (int p = 0; p < O::kParts; ++p) part[p][j].w[i] = pack_part<O::kHalf>(f[j], g[j]);
            }
        }
    }
#pragma unroll
    for (int p = 0; p < O::kParts; ++p)
#pragma unroll
        for (int j = 0; j < kQuad; ++j) to[p * kChunks * kTile + j * kQuads] = part[p][j];
}

template <bool kHalf>
__device__ __forceinline__ f32x4 multiply(const Piece &a, const Piece &b, f32x4 c)
{
    if constexpr (kHalf) {
        typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
}

// D, X: types of dy and x.  Four waves of 64 x 64 outputs; x's columns are the rows
// of the matrix unit's result, so a lane has four neighbouring outputs.
template <typename D, typename X, bool kExact>
__global__ __launch_bounds__(kThreads, 2) void eb_gradient_tile(GradientArgs a)
{
    constexpr bool kFp8D = std::is_same_v<D, Fp8>, kFp8X = std::is_same_v<X, Fp8>, kScaled = kFp8D || kFp8X;
    constexpr bool kHalf = !std::is_same_v<D, Bf16> && !std::is_same_v<X, Bf16>;
    constexpr bool kShift = kHalf && kScaled; // scales are divided by a power of two
    using OD = Operand<D, kFp8D && !kFp8X, kHalf, kExact>;
    using OX = Operand<X, kFp8X, kHalf, kExact>;
    __shared__ Piece of_dy[OD::kParts][kChunks][kTile], of_x[OX::kParts][kChunks][kTile];
    __shared__ int32_t row_of[2][kSlots]; // of x; -1: the slot adds nothing
    __shared__ float scale_of[2][kSlots];
    __shared__ int most_of[2]; // the exponent of the largest scale of a step

    uint32_t at = blockIdx.x;
    const int k_tile = at % a.k_tiles;
    at /= a.k_tiles;
    const int n_tile = at % a.n_tiles;
    at /= a.n_tiles;
    const int split = at % a.splits, e = at / a.splits;
    int begin = 0, end = a.M;
    if (a.offsets) {
        begin = min(max(eb_detail::scalar_load(a.offsets + e), 0), a.M);
        end = min(max(eb_detail::scalar_load(a.offsets + e + 1), begin), a.M);
    }
    const int64_t each = (((int64_t)end - begin + a.splits - 1) / a.splits + kSlots - 1) / kSlots * kSlots;
    begin = (int)min(begin + split * each, (int64_t)end);
    end = (int)min(begin + each, (int64_t)end);

    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
    const int chunk = t / kQuads, quad = t % kQuads;
    const int n0 = n_tile * kTile, k0 = k_tile * kTile;

    // A slot's row of x, and its scale, a step ahead of the operands themselves.
    auto row_at = [&](int64_t m) {
        if (m >= end) return -1;
        const int r = a.tokens ? a.tokens[m] : (int)m;
        return r >= 0 && r < a.x_rows ? r : -1;
    };
    auto scale_at = [&](int64_t m, int row) {
        float s = row < 0 ? 0.f : 1.f;
        if (row >= 0 && kFp8D) s = a.dy_scales.p[n_tile * a.dy_scales.ld + m];
        if (row >= 0 && kFp8X) s *= a.x_scales.p[k_tile * a.x_scales.ld + row];
        return s;
    };
    // By the first wave, whose lanes have a slot each.
    auto put = [&](int of, int row, float s) {
        row_of[of][t] = row;
        if constexpr (kScaled) scale_of[of][t] = s;
        if constexpr (kShift) {
            const int bits = magnitude(s), most = max_lanes<kWave>(bits < 0x7F800000 ? bits >> 23 : 0);
            if (t == 0) most_of[of] = most;
        }
    };
    uint32_t raw_dy[8][OD::kWords], raw_x[8][OX::kWords];
    auto load = [&](int64_t m, const int32_t *rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = rows[chunk * 8 + i];
#pragma unroll
            for (int j = 0; j < OD::kWords; ++j) raw_dy[i][j] = 0;
#pragma unroll
            for (int j = 0; j < OX::kWords; ++j) raw_x[i][j] = 0;
            if (row >= 0) {
                load_quad<D>(a.dy + (m + chunk * 8 + i) * a.lddy, n0 + quad * kQuad, a.N, raw_dy[i]);
                load_quad<X>(a.x + row * a.ldx, k0 + quad * kQuad, a.K, raw_x[i]);
            }
        }
    };

    f32x4 sum[4][4] = {}; // [columns of dy][columns of x]
    const int wk = wave % 2, wn = wave / 2;
    constexpr int kMostLeft = 5; // 2^6 above the largest e4m3 value, 2^15 and less
    int next_row = -1, shift = -200; // below any scale's exponent
    if (begin < end) {
        if (t < kSlots) {
            const int row = row_at(begin + t);
            put(0, row, scale_at((int64_t)begin + t, row));
            next_row = row_at((int64_t)begin + kSlots + t);
        }
        __syncthreads();
        load(begin, row_of[0]);
    }
    int turn_of = 0;
    for (int64_t m = begin; m < end; m += kSlots, turn_of ^= 1) {
        float next_scale = 0.f;
        const int row = next_row;
        if (kScaled && t < kSlots) next_scale = scale_at(m + kSlots + t, row);
        float scale[8];
        if constexpr (kScaled) {
#pragma unroll
            for (int i = 0; i < 8; ++i) scale[i] = scale_of[turn_of][chunk * 8 + i];
        }
        if constexpr (kShift) {
            // 448 S / 2^shift stays below 2^15; a new shift leaves room for S to grow 16 times.
            const int most = __builtin_amdgcn_readfirstlane(most_of[turn_of]) - 127;
            if (most - shift > kMostLeft) {
                const int to = most - kMostLeft + 4;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum[i][j][r] = ldexpf(sum[i][j][r], shift - to);
                shift = to;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) scale[i] = ldexpf(scale[i], -shift);
        }
        __syncthreads(); // the last step's operands have been read
        turn<OD>(raw_dy, scale, &of_dy[0][chunk][quad]);
        turn<OX>(raw_x, scale, &of_x[0][chunk][quad]);
        if (t < kSlots) {
            put(turn_of ^ 1, row, next_scale);
            next_row = row_at(m + 2 * kSlots + t);
        }
        __syncthreads();
        if (m + kSlots < end) load(m + kSlots, row_of[turn_of ^ 1]);
#pragma unroll
        for (int s = 0; s < kSlots / 32; ++s) {
            const int c = s * 4 + lane / 16;
            Piece x[OX::kParts][4], y[OD::kParts][4];
#pragma unroll
            for (int p = 0; p < OX::kParts; ++p)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[p][j] = of_x[p][c][j * kQuads + wk * 16 + lane % 16];
#pragma unroll
            for (int p = 0; p < OD::kParts; ++p)
#pragma unroll
                for (int j = 0; j < 4; ++j) y[p][j] = of_dy[p][c][j * kQuads + wn * 16 + lane % 16];
#pragma unroll
            for (int q = 0; q < OD::kParts; ++q)
#pragma unroll
                for (int p = 0; p < OX::kParts; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) sum[i][j] = multiply<kHalf>(x[p][j], y[q][i], sum[i][j]);
        }
    }

    // Lane l has column l % 16 of the unit's result (dy's) and rows 4 (l / 16) + r.
    float *partial = a.partial ? a.partial + ((int64_t)split * a.E + e) * a.N * a.K : nullptr;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = n0 + wn * 64 + lane % 16 * kQuad + i;
        if (n >= a.N) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int k = k0 + wk * 64 + (lane / 16 * 4 + r) * kQuad;
            if (k >= a.K) continue;
            float v[kQuad];
#pragma unroll
            for (int j = 0; j < kQuad; ++j) v[j] = kShift ? ldexpf(sum[i][j][r], shift) : sum[i][j][r];
            const int left = a.K - k;
            if (partial) {
                float *to = partial + (int64_t)n * a.K + k;
                if (left >= kQuad) {
                    const i32x4_any w = {__float_as_int(v[0]), __float_as_int(v[1]), __float_as_int(v[2]), __float_as_int(v[3])};
                    *(i32x4_any *)to = w;
                } else {
                    for (int j = 0; j < left; ++j) to[j] = j == 0 ? v[0] : j == 1 ? v[1] : v[2];
                }
                continue;
            }
            const int64_t place = ((int64_t)e * a.N + n) * a.lddw + k;
#pragma unroll
            for (int j = 0; j < kQuad; ++j) {
                if (j >= left) break;
                if (a.out_type == EB_F32) {
                    float *to = (float *)a.dw + place + j;
                    *to = a.accumulate ? *to + v[j] : v[j];
                } else if (a.out_type == EB_F16) {
                    _Float16 *to = (_Float16 *)a.dw + place + j;
                    *to = (_Float16)(a.accumulate ? (float)*to + v[j] : v[j]);
                } else {
                    __bf16 *to = (__bf16 *)a.dw + place + j;
                    *to = (__bf16)(a.accumulate ? (float)*to + v[j] : v[j]);
                }
            }
        }
    }
}

} // namespace eb_gradient
