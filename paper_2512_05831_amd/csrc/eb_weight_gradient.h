// eb_weight_gradient (include/eb_train.h), its kernel: for every expert
//
//   dw[n, k] = sum over its slots m of dy[m, n] x[token of m, k]
//
// with the 16-bit matrix unit.  Both operands lie with the slots one below the other,
// while the unit wants eight slots of one column in a lane.  They are copied as they lie
// from global memory straight into LDS, the next step's while this one is multiplied,
// and read from there by the instructions that turn 8 (of 16 bits: 4) rows of 16
// columns on the way.  8-bit values become 16-bit ones in the wave that read them.
//   A workgroup has 256 columns of one operand (the "own" one: a wave has 64 of them
// to itself) by 128 of the other (the "shared" one, which all four waves read), so what
// is costly to make of a value is made once if the own operand has it.
//   A slot's scales (of dy and of x) go into the own operand as their product S, one
// number for a slot and 128 own columns; so that the shared one, e4m3 or 16 bits,
// enters exactly, and where dy and x both have scales a workgroup's shared columns are
// one block of them.  Scaled values have up to 28 bits and take several 16-bit parts,
// each multiplied with the shared operand:
//   beside e4m3 or fp16, two parts in fp16 (22 bits).  Their range is short, so S (in two
//     parts too) is divided by a power of two that keeps the largest S so far in [2^11,
//     2^14), and the e4m3 value by 2^8 (exactly: it is 2^-17 and more).  What fp16, whose
//     numbers lie 2^-24 apart and more, cannot hold of S and of the products is then below
//     2^-34 of the largest product.  Where the power grows the sums are brought to the new one
//     (exactly), and the outputs multiplied by the last;
//   beside bfloat16, three parts in that (24 bits), for bfloat16 outputs two (16 bits, a
//     512th of those outputs' own rounding; 8192 slots by 32 experts of 512 x 1024 take 40 us,
//     in one part, whose error is that rounding's size again, 33).
//   In LDS the 16-byte pieces of a row are permuted with its number (what a lane copies
// goes where its number says, so it is the global addresses that are permuted): the
// rows that an instruction reads at a time then lie in different banks.
#pragma once

#include <type_traits>

#include "eb_train.h"

namespace eb_gradient {

using namespace eb_train;

constexpr int kThreads = 256;
constexpr int kOwnTile = 256; // columns of the own operand, of a workgroup
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct GradientArgs {
    const char *own, *shared;
    Scales own_scales, shared_scales;
    const int32_t *tokens, *offsets;
    void *dw;
    float *partial;                 // [splits][E][N, K], or NULL
    int64_t own_ld, shared_ld;      // in bytes
    int64_t x_rows, lddw;
    int32_t own_cols, shared_cols;
    int32_t M, E, N, K;
    int32_t own_tiles, shared_tiles, splits;
    int32_t out_type;
    bool accumulate;
};

struct alignas(16) Piece { // eight slots of a column, 16 bits each
    uint32_t w[4];
};
struct alignas(8) Bytes { // 8 bits each
    uint32_t w[2];
};

// Which operand is the own one, and how it enters the unit.
template <typename D, typename X, bool kExact>
struct Shape {
    static constexpr bool kHalf = !std::is_same_v<D, Bf16> && !std::is_same_v<X, Bf16>; // the unit takes fp16, else bfloat16
    using Unit = std::conditional_t<kHalf, _Float16, Bf16>;
    // dy, but where x has scales and dy has none, or x alone is of another type than the unit's.
    static constexpr bool kOwnX = !std::is_same_v<D, Fp8> && !std::is_same_v<X, Unit>;
    using Own = std::conditional_t<kOwnX, X, D>;
    using Shared = std::conditional_t<kOwnX, D, X>;
    static constexpr bool kScaled = std::is_same_v<Own, Fp8>;
    static constexpr bool kBoth = kScaled && std::is_same_v<Shared, Fp8>;
    static constexpr bool kShift = kScaled && kHalf;
    static constexpr bool kAsItIs = std::is_same_v<Own, Unit>;
    static constexpr int kParts = kAsItIs ? 1 : kHalf || !kScaled || !kExact ? 2 : 3; // (fp16 values are exact in two of bfloat16)
    using OwnPiece = std::conditional_t<kScaled, Bytes, Piece>;
    static constexpr int kSlots = kScaled ? 64 : 32; // of a step
};

constexpr int kQuad = 4;                    // neighbouring outputs of a lane
constexpr int kHalves = kOwnTile / kBlock;  // blocks of scales of the own operand
constexpr int kInfos = 3;                   // steps whose slots are known at a time

// One step of an operand in LDS, and how it gets there and out of there.
template <typename T, int kColumns, int kSlots>
struct Panel {
    static constexpr uint32_t kRow = kColumns * sizeof(T), kPieces = kRow / 16; // of a slot
    static constexpr uint32_t kRows = kThreads / kPieces;                       // of a copy by all threads
    static constexpr int kCopies = kSlots / kRows;
    static_assert(kSlots % kRows == 0, "whole copies");
    alignas(16) char bytes[kSlots * kRow];

    // The piece of a row that lies in place `at` of it.
    static __device__ __forceinline__ uint32_t piece_of(uint32_t row, uint32_t at)
    {
        return at ^ (sizeof(T) == 1 ? swap_of(row) : 2 * swap_of(row));
    }
    // 16 rows of 8 bits, one piece each, and 8 of 16 bits, two, fill a line of the banks.
    static __device__ __forceinline__ uint32_t swap_of(uint32_t row)
    {
        if constexpr (sizeof(T) == 1) return row / (16 / kPieces) % kPieces;
        else return kPieces >= 16 ? row % 4 | row / 8 % 2 * 4 : row / 2 % 2 | row / 8 % 2 * 2;
    }

    // Where a lane reads from for column tile 0; for tile i that ^ i * kTile.
    static constexpr uint32_t kTile = 16 * sizeof(T);
    static __device__ __forceinline__ uint32_t first_of(uint32_t lane)
    {
        const uint32_t g = lane / 16, in = lane % 16;
        if constexpr (sizeof(T) == 1) {
            const uint32_t row = 8 * g + in / 2;
            return row * kRow + swap_of(row) * 16 + in % 2 * 8;
        } else {
            const uint32_t row = 8 * g + in / 4; // and the fourth from it, of the same swap
            return row * kRow + swap_of(row) * 32 + in % 4 * 8;
        }
    }

    // Columns 16 tile .. + 15 of slots 8 g .. 8 g + 7, g = step / 8 + lane / 16: column lane % 16.
    __device__ __forceinline__ std::conditional_t<sizeof(T) == 1, Bytes, Piece> read(int step, uint32_t first, uint32_t tile) const
    {
        typedef __attribute__((address_space(3))) char Lds;
        const auto from = (const Lds *)bytes + ((first ^ tile * kTile) + step * kRow);
        if constexpr (sizeof(T) == 1) {
            typedef int i32x2 __attribute__((ext_vector_type(2)));
            return __builtin_bit_cast(Bytes, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2 *)from));
        } else {
            typedef short i16x4 __attribute__((ext_vector_type(4)));
            const i16x4 v[2] = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)from),
                                __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(from + 4 * kRow))};
            return __builtin_bit_cast(Piece, v);
        }
    }
};

__device__ const i32x4 kZeros = {0, 0, 0, 0};

// The first `left` bytes (below 16) at an address of any alignment, zeros behind them.
__device__ __forceinline__ i32x4 load_some(const char *at, uint32_t left)
{
    uint32_t w[4] = {};
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i)
        if (2 * i < left) w[i / 2] |= (uint32_t)((const uint16_t *)at)[i] << i % 2 * 16;
    return i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}

// 16 bytes without the first `n` (even, below 16), zeros behind the others.
__device__ __forceinline__ i32x4 drop_bytes(i32x4 v, uint32_t n)
{
    uint32_t w[5] = {(uint32_t)v[0], (uint32_t)v[1], (uint32_t)v[2], (uint32_t)v[3], 0};
    if (n & 8) w[0] = w[2], w[1] = w[3], w[2] = 0, w[3] = 0;
    if (n & 4) w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_alignbyte(w[i + 1], w[i], n & 2);
    return i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}

__device__ __forceinline__ Piece widened(const Bytes &b)
{
    Piece p;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        p.w[i] = __builtin_bit_cast(uint32_t, i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b.w[i / 2], 1.f, true)
                                                    : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b.w[i / 2], 1.f, false));
    return p;
}

template <bool kHalf>
__device__ __forceinline__ f32x4 multiply(const Piece &a, const Piece &b, f32x4 c)
{
    if constexpr (kHalf)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// An e4m3 value beside fp16 scales counts these, and its scale as many times more.
constexpr int kOwnShift = 8;
constexpr float kOwnUnit = 1.f / (1 << kOwnShift);

// Scales of the eight slots of a lane, as the own operand's parts are made with them.
template <bool kHalf>
struct EightScales;
template <>
struct EightScales<true> {
    f16x2 first[4], rest[4]; // S rounded to fp16, and what that leaves
};
template <>
struct EightScales<false> {
    float s[8];
};

// The own operand's parts, made of a piece in LDS and taken one after the other.
template <typename S, typename Take>
__device__ __forceinline__ void each_part(const typename S::OwnPiece &piece, const EightScales<S::kHalf> &scale, Take &&take)
{
    if constexpr (S::kAsItIs) {
        take(piece);
    } else if constexpr (S::kShift) {
        Piece first, rest;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f16x2 q = i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(piece.w[i / 2], kOwnUnit, true)
                                  : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(piece.w[i / 2], kOwnUnit, false);
            const f16x2 v = q * scale.first[i];
            first.w[i] = __builtin_bit_cast(uint32_t, v);
            // What v's rounding left of q * first (exactly, or to 2^-25), and q * rest, rounded once.
            const f16x2 left = __builtin_elementwise_fma(q, scale.first[i], -v);
            rest.w[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(q, scale.rest[i], left));
        }
        take(first);
        take(rest);
    } else {
        float f[kEach];
        if constexpr (S::kScaled) {
            Raw<Fp8> raw;
            __builtin_memcpy(&raw, &piece, 8);
            widen8(raw, f);
#pragma unroll
            for (int i = 0; i < kEach; ++i) f[i] *= scale.s[i];
        } else {
            Raw<_Float16> raw;
            __builtin_memcpy(&raw, &piece, 16);
            widen8(raw, f);
        }
#pragma unroll
        for (int p = 0; p < S::kParts; ++p) {
            Piece part;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t w = pack_bf16(f[2 * i], f[2 * i + 1]);
                part.w[i] = w;
                f[2 * i] -= __uint_as_float(w << 16);
                f[2 * i + 1] -= __uint_as_float(w & 0xFFFF0000u);
            }
            take(part);
        }
    }
}

// Workgroups are dealt to the 8 XCDs in turn.  Each takes runs of tiles that have the
// same own columns, and so share them in its L2, the runs in turn: every expert's tiles
// spread over the XCDs, whatever its slots.
__device__ __forceinline__ uint32_t tile_in_order(uint32_t index, uint32_t count, uint32_t run)
{
    constexpr uint32_t kXcds = 8;
    const uint32_t whole = count / kXcds / run * (kXcds * run);
    if (index >= whole) return index;
    const uint32_t xcd = index % kXcds, nth = index / kXcds;
    return (nth / run * kXcds + xcd) * run + nth % run;
}

template <typename T>
__device__ __forceinline__ void write_out(T *to, bool accumulate, float v)
{
    *to = (T)(accumulate ? (float)*to + v : v);
}

// Four neighbouring outputs from `place` of dw on, `left` of them there.
__device__ __forceinline__ void write_values(const GradientArgs &a, int64_t place, int left, const float *v)
{
    if (left >= kQuad && !a.accumulate) {
        if (a.out_type == EB_F32) {
            const i32x4_any w = {__float_as_int(v[0]), __float_as_int(v[1]), __float_as_int(v[2]), __float_as_int(v[3])};
            *(i32x4_any *)((float *)a.dw + place) = w;
        } else {
            const bool half = a.out_type == EB_F16;
            const i32x2_any w = {(int)(half ? pack16((_Float16)v[0], (_Float16)v[1]) : pack_bf16(v[0], v[1])),
                                 (int)(half ? pack16((_Float16)v[2], (_Float16)v[3]) : pack_bf16(v[2], v[3]))};
            *(i32x2_any *)((uint16_t *)a.dw + place) = w;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < kQuad; ++j) {
        if (j >= left) break;
        if (a.out_type == EB_F32) write_out((float *)a.dw + place + j, a.accumulate, v[j]);
        else if (a.out_type == EB_F16) write_out((_Float16 *)a.dw + place + j, a.accumulate, v[j]);
        else write_out((__bf16 *)a.dw + place + j, a.accumulate, v[j]);
    }
}

// Those of row n from column k on, or a split's share of them.
__device__ __forceinline__ void write_quad(const GradientArgs &a, float *partial, int e, int n, int k, const float *v)
{
    const int left = a.K - k;
    if (!partial) return write_values(a, ((int64_t)e * a.N + n) * a.lddw + k, left, v);
    float *to = partial + (int64_t)n * a.K + k;
    if (left >= kQuad) {
        const i32x4_any w = {__float_as_int(v[0]), __float_as_int(v[1]), __float_as_int(v[2]), __float_as_int(v[3])};
        *(i32x4_any *)to = w;
    } else {
#pragma unroll
        for (int j = 0; j < kQuad; ++j)
            if (j < left) to[j] = v[j];
    }
}

// kDirect: 16-bit operands lie so that 16 bytes can be copied to LDS at a time (8-bit
// ones always do); else they go through registers, in narrow tiles, whose sums leave
// room for them (12000 slots by 2047 x 2047, fp16 by 8 bits: 537 us in wide ones, 249 in
// narrow ones; bf16 270 and 293; by 2048 x 2048, copied, 191 and 133).
template <typename D, typename X, bool kExact, bool kDirect, int kSharedTile>
__global__ __launch_bounds__(kThreads, kSharedTile == 64 && kDirect ? 3 : 2) void eb_gradient_tile(GradientArgs a)
{
    using S = Shape<D, X, kExact>;
    using Own = typename S::Own;
    using Shared = typename S::Shared;
    constexpr int kSlots = S::kSlots;
    using OwnPanel = Panel<Own, kOwnTile, kSlots>;
    using SharedPanel = Panel<Shared, kSharedTile, kSlots>;
    constexpr bool kOwnDirect = kDirect || sizeof(Own) == 1, kSharedDirect = kDirect || sizeof(Shared) == 1;
    constexpr int kSharedTiles = kSharedTile / 16, kOwnTiles = kOwnTile / 64; // 16 x 16 tiles of a wave
    // What is copied to while another step is read is a variable of its own: the
    // compiler then sees that those reads need not wait for the copies.
    __shared__ OwnPanel own_even, own_odd;
    __shared__ SharedPanel shared_even, shared_odd;
    __shared__ int64_t offset_of[kInfos][kSlots]; // of a slot's row of x; -1: the slot adds nothing
    __shared__ std::conditional_t<S::kHalf, _Float16, float> first_of[kInfos][kHalves][kSlots], rest_of[kInfos][kHalves][kSlots];
    __shared__ int shift_of[kInfos][kHalves];

    uint32_t at = tile_in_order(blockIdx.x, gridDim.x, a.shared_tiles);
    const int shared_tile = at % a.shared_tiles;
    at /= a.shared_tiles;
    const int own_tile = at % a.own_tiles;
    at /= a.own_tiles;
    const int split = at % a.splits, e = at / a.splits;
    int begin = 0, end = a.M;
    if (a.offsets) {
        begin = min(max(eb_detail::scalar_load(a.offsets + e), 0), a.M);
        end = min(max(eb_detail::scalar_load(a.offsets + e + 1), begin), a.M);
    }
    const int64_t each = (((int64_t)end - begin + a.splits - 1) / a.splits + kSlots - 1) / kSlots * kSlots;
    begin = (int)min(begin + split * each, (int64_t)end);
    end = a.x_rows == 0 ? begin : (int)min(begin + each, (int64_t)end);

    const int t = threadIdx.x, lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
    const int own0 = own_tile * kOwnTile, shared0 = shared_tile * kSharedTile;

    // A step's slots: where their rows of x are, and their scales; by the first threads
    // (kSlots for each block of own columns), two steps ahead.
    const bool informs = t < kHalves * kSlots;
    const int slot = threadIdx.x % kSlots, half = threadIdx.x / kSlots;
    // Loads whose values wait until they are needed, from places that are there (a step
    // has slots, and x rows); what they say of slots that are not is left out then.
    auto token_at = [&](int64_t m) { return a.tokens ? a.tokens[min(m, (int64_t)end - 1)] : (int)min(m, (int64_t)end); };
    auto row_of = [&](int64_t m, int token) { return m < end && token >= 0 && token < a.x_rows ? token : -1; };
    const int64_t block = min((int64_t)own_tile * kHalves + half, ((int64_t)a.own_cols - 1) / kBlock);
    float own_scale = 0.f, shared_scale = 1.f;
    auto load_scales = [&](int64_t m, int row) {
        if constexpr (S::kScaled) own_scale = a.own_scales.p[block * a.own_scales.ld + (S::kOwnX ? max(row, 0) : min(m, (int64_t)end - 1))];
        if constexpr (S::kBoth) shared_scale = a.shared_scales.p[shared0 / kBlock * a.shared_scales.ld + max(row, 0)];
    };
    int next_shift = -200; // below any scale's exponent
    auto put = [&](int of, int row) {
        if (half == 0) offset_of[of][slot] = row < 0 ? -1 : row * (S::kOwnX ? a.own_ld : a.shared_ld);
        if constexpr (S::kScaled) {
            float s = row < 0 ? 0.f : own_scale * shared_scale;
            if constexpr (S::kShift) {
                // S / 2^shift stays below 2^14, and 448 kOwnUnit times that below 2^15; a new
                // shift leaves room for S to grow 4 times.
                constexpr int kMostLeft = 5 + kOwnShift, kRoom = 2;
                static_assert(kSlots == kWave, "a wave has a step's scales of a block");
                const int bits = magnitude(s), most = max_lanes<kWave>(bits < 0x7F800000 ? bits >> 23 : 0) - 127;
                if (most - next_shift > kMostLeft) next_shift = most - kMostLeft + kRoom;
                if (slot == 0) shift_of[of][half] = next_shift;
                s = ldexpf(s, -next_shift);
                const _Float16 first = (_Float16)s;
                first_of[of][half][slot] = first;
                rest_of[of][half][slot] = (_Float16)(s - (float)first);
            } else {
                first_of[of][half][slot] = s;
            }
        }
    };

    // Copies of a step that begins with slot m, 16 bytes a lane.  Direct ones take 16
    // bytes of zeros in place of what is not there.
    const auto zeros = (const char *)&kZeros;
    const uint32_t thread = t;
    i32x4 own_raw[kOwnDirect ? 1 : OwnPanel::kCopies], shared_raw[kSharedDirect ? 1 : SharedPanel::kCopies];
    // dy's rows follow each other: where the thread's first one is from a step's start on.
    constexpr uint32_t kRowsOfDy = S::kOwnX ? SharedPanel::kRows : OwnPanel::kRows;
    const int64_t dy_ld = S::kOwnX ? a.shared_ld : a.own_ld, of_dy = thread / (kThreads / kRowsOfDy) * dy_ld;
    // Bytes before a piece that are read with it, where it ends past its row.
    auto back_of = [](uint32_t byte, uint32_t left) { return byte < left && byte + 16 > left ? byte + 16 - left : 0; };
    auto copy = [&](auto &panel, auto direct, auto of_x, i32x4 *raw, const char *base, uint32_t left, int64_t m, int of, bool few) {
        using P = std::remove_reference_t<decltype(panel)>;
        const char *dy = base + m * dy_ld;
#pragma unroll
        for (int p = 0; p < P::kCopies; ++p) {
            const uint32_t row = p * P::kRows + thread / P::kPieces, byte = P::piece_of(row, thread % P::kPieces) * 16;
            const int64_t x = offset_of[of][row];
            const char *from = decltype(of_x)::value ? base + x : dy + p * (int64_t)P::kRows * dy_ld + of_dy;
            from += byte;
            if constexpr (decltype(direct)::value) {
                from = x < 0 || byte >= left ? zeros : from;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                                 (__attribute__((address_space(3))) void *)(panel.bytes + (p * kThreads + wave * kWave) * 16), 16, 0, 0);
            } else {
                // Whole 16 bytes in any case, so that no load waits for another: a row's last
                // ones together with what is before them, which is dropped when they are stored.
                const bool there = x >= 0 && byte < left;
                if (few) raw[p] = load_some(there ? from : zeros, there ? left - byte : 0);
                else raw[p] = *(const i32x4_any *)(there ? from - back_of(byte, left) : zeros);
            }
        }
    };
    auto left_of = [](int cols, int first, int width, int size) { return (uint32_t)(min(cols - first, width) * size); };
    const uint32_t own_left = left_of(a.own_cols, own0, kOwnTile, sizeof(Own)), shared_left = left_of(a.shared_cols, shared0, kSharedTile, sizeof(Shared));
    const bool own_few = a.own_cols < 8, shared_few = a.shared_cols < 8; // rows of less than 16 bytes
    auto copy_step = [&](auto &own, auto &shared, int64_t m, int of) {
        copy(own, std::bool_constant<kOwnDirect>(), std::bool_constant<S::kOwnX>(), own_raw, a.own + (int64_t)own0 * sizeof(Own), own_left, m, of, own_few);
        copy(shared, std::bool_constant<kSharedDirect>(), std::bool_constant<!S::kOwnX>(), shared_raw, a.shared + (int64_t)shared0 * sizeof(Shared),
             shared_left, m, of, shared_few);
    };
    auto store = [&](auto &panel, const i32x4 *raw, uint32_t left, bool few) {
        using P = std::remove_reference_t<decltype(panel)>;
#pragma unroll
        for (int p = 0; p < P::kCopies; ++p) {
            const uint32_t row = p * P::kRows + thread / P::kPieces, back = few ? 0 : back_of(P::piece_of(row, thread % P::kPieces) * 16, left);
            i32x4 v = raw[p];
            if (__any(back != 0)) v = drop_bytes(v, back);
            *(i32x4 *)(panel.bytes + (p * kThreads + thread) * 16) = v;
        }
    };
    auto store_step = [&](auto &own, auto &shared) { // what went through registers
        if constexpr (!kOwnDirect) store(own, own_raw, own_left, own_few);
        if constexpr (!kSharedDirect) store(shared, shared_raw, shared_left, shared_few);
    };

    // x's columns are the rows of the unit's result, of which a lane has four neighbours.
    f32x4 sum[kSharedTiles][kOwnTiles] = {};
    int shift = -200;
    const int own_half = wave * 64 / kBlock;
    const uint32_t shared_first = SharedPanel::first_of(lane), own_first = OwnPanel::first_of(lane) ^ wave * kOwnTiles * OwnPanel::kTile;
    auto multiply_step = [&](const OwnPanel &own, const SharedPanel &shared, int of) {
        if constexpr (S::kShift) {
            const int to = __builtin_amdgcn_readfirstlane(shift_of[of][own_half]);
            if (to != shift) {
#pragma unroll
                for (int i = 0; i < kSharedTiles; ++i)
#pragma unroll
                    for (int j = 0; j < kOwnTiles; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum[i][j][r] = ldexpf(sum[i][j][r], shift - to);
                shift = to;
            }
        }
#pragma unroll
        for (int s = 0; s < kSlots; s += 32) {
            Piece other[kSharedTiles];
#pragma unroll
            for (int i = 0; i < kSharedTiles; ++i) {
                if constexpr (sizeof(Shared) == 1) other[i] = widened(shared.read(s, shared_first, i));
                else other[i] = shared.read(s, shared_first, i);
            }
            EightScales<S::kHalf> scale;
            const int c = s + lane / 16 * 8;
            if constexpr (S::kShift) {
                __builtin_memcpy(scale.first, &first_of[of][own_half][c], 16);
                __builtin_memcpy(scale.rest, &rest_of[of][own_half][c], 16);
            } else if constexpr (S::kScaled) {
                __builtin_memcpy(scale.s, &first_of[of][own_half][c], 32);
            }
#pragma unroll
            for (int j = 0; j < kOwnTiles; ++j) {
                each_part<S>(own.read(s, own_first, j), scale, [&](const Piece &part) {
#pragma unroll
                    for (int i = 0; i < kSharedTiles; ++i)
                        sum[i][j] = S::kOwnX ? multiply<S::kHalf>(part, other[i], sum[i][j]) : multiply<S::kHalf>(other[i], part, sum[i][j]);
                });
                // The sums stay where they are: else the compiler moves them about, and runs out of registers.
#pragma unroll
                for (int i = 0; i < kSharedTiles; ++i) asm volatile("" : "+v"(sum[i][j]));
            }
        }
    };

    int row = -1, token = -1, of = 0;
    // A step: the copies of the one after it go out, then it is multiplied.
    auto step = [&](auto &own, auto &shared, auto &next_own, auto &next_shared, int64_t m) {
        __builtin_amdgcn_s_waitcnt(0x0F70); // vmcnt(0): this wave's copies, which a barrier does not wait for
        __syncthreads();                    // all its copies are there, and the other step's have been read
        const int next = of == kInfos - 1 ? 0 : of + 1, after = next == kInfos - 1 ? 0 : next + 1;
        if (informs) {
            put(after, row);
            row = row_of(m + 3 * kSlots + slot, token);
            load_scales(m + 3 * kSlots + slot, row);
            token = token_at(m + 4 * kSlots + slot);
        }
        const bool more = m + kSlots < end;
        if (more) copy_step(next_own, next_shared, m + kSlots, next);
        multiply_step(own, shared, of);
        if (more) store_step(next_own, next_shared);
        of = next;
    };
    if (begin < end) {
        if (informs) {
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                const int64_t m = (int64_t)begin + i * kSlots + slot;
                row = row_of(m, token_at(m));
                load_scales(m, row);
                if (i < 2) put(i, row);
            }
            token = token_at((int64_t)begin + 3 * kSlots + slot);
        }
        __syncthreads();
        copy_step(own_even, shared_even, begin, 0);
        store_step(own_even, shared_even);
        for (int64_t m = begin; m < end; m += 2 * kSlots) {
            step(own_even, shared_even, own_odd, shared_odd, m);
            if (m + kSlots < end) step(own_odd, shared_odd, own_even, shared_even, m + kSlots);
        }
    }

    // Lane l has column l % 16 of the unit's result (dy's) and rows 4 (l / 16) + r (x's).
    float *partial = a.partial ? a.partial + ((int64_t)split * a.E + e) * a.N * a.K : nullptr;
#pragma unroll
    for (int j = 0; j < kOwnTiles; ++j)
#pragma unroll
        for (int i = 0; i < kSharedTiles; ++i) {
            const int own = own0 + wave * 64 + j * 16, shared = shared0 + i * 16;
            const int n = (S::kOwnX ? shared : own) + lane % 16, k = (S::kOwnX ? own : shared) + lane / 16 * kQuad;
            if (n >= a.N || k >= a.K) continue;
            float v[kQuad];
#pragma unroll
            for (int r = 0; r < kQuad; ++r) v[r] = S::kShift ? ldexpf(sum[i][j][r], shift + kOwnShift) : sum[i][j][r];
            write_quad(a, partial, e, n, k, v);
        }
}

struct Choice {
    void *kernel;
    bool own_x;
};

template <typename D, typename X, int kSharedTile>
Choice choice_of(bool exact, bool direct)
{
    using S = Shape<D, X, true>;
    constexpr bool kTwoForms = S::kParts == 3; // else both are the same
    if constexpr (!kTwoForms) exact = true;
    if constexpr (sizeof(D) == 1 && sizeof(X) == 1) direct = true;
    if (direct && exact) return {(void *)eb_gradient_tile<D, X, true, true, kSharedTile>, S::kOwnX};
    if constexpr (kTwoForms)
        if (direct) return {(void *)eb_gradient_tile<D, X, false, true, kSharedTile>, S::kOwnX};
    if constexpr (kSharedTile == 64 && (sizeof(D) == 2 || sizeof(X) == 2)) {
        if (exact) return {(void *)eb_gradient_tile<D, X, true, false, kSharedTile>, S::kOwnX};
        if constexpr (kTwoForms) return {(void *)eb_gradient_tile<D, X, false, false, kSharedTile>, S::kOwnX};
    }
    return {};
}

template <typename D>
Choice choice_of(int32_t x_type, bool exact, bool direct, bool narrow)
{
    if (narrow)
        return x_type == EB_FP8   ? choice_of<D, Fp8, 64>(exact, direct)
               : x_type == EB_F16 ? choice_of<D, _Float16, 64>(exact, direct)
                                  : choice_of<D, Bf16, 64>(exact, direct);
    return x_type == EB_FP8   ? choice_of<D, Fp8, 128>(exact, true)
           : x_type == EB_F16 ? choice_of<D, _Float16, 128>(exact, true)
                              : choice_of<D, Bf16, 128>(exact, true);
}

// By dy's type, each in a source of its own.
Choice choice_fp8(int32_t x_type, bool exact, bool direct, bool narrow);
Choice choice_f16(int32_t x_type, bool exact, bool direct, bool narrow);
Choice choice_bf16(int32_t x_type, bool exact, bool direct, bool narrow);

} // namespace eb_gradient
