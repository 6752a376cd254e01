// eb_expert_product for many slots per expert: bound by the matrix units and, on
// the way to them, by the power they may draw.
//
// A workgroup takes kTokens16 * kAcrossT * 16 slots of an expert by kRows16 * 64
// weight rows, a wave kTokens16 x kRows16 tiles of 16 x 16, four waves side by side
// along the rows.  A block of 128 of both operands (and the tokens' scales) goes from global
// memory straight into LDS, the next block's while this one is multiplied, and
// one barrier parts the two.  Where there are few tiles it is the time of a block,
// not the rate, that counts: 2048 slots by 1000 x 1512, fp32 out, 15.8 us in tiles of 32 x
// 256, 12.2 in 32 x 128, two a compute unit, 13.6 in 32 x 64.
//   Four waves (kAcrossT 1): the tokens are double-buffered; the weights are a
// wave's own and single: once it has them in its registers it sends for the next
// block's.  That is 66 KB for 128 slots, so a compute unit holds two workgroups,
// and one's epilogue runs beside the other's products.
//   Eight waves (kAcrossT 2, 256 slots): two stages of both operands, 134 KB, one
// workgroup a compute unit, two thirds of the copies for the same products.
//   In LDS a row is its 128 bytes, chunk c of 16 bytes at place c ^ (row % 8): the
// eight lanes that an LDS access serves at a time then read eight different
// chunks of the 128-byte line of banks.  (The place in LDS follows from the lane,
// so it is the global addresses that are permuted.)
//
// Measured on random normal values in long runs: 16384 slots by 4096 x 3328 in the
// 8-bit unit 203 us, 2.2 PFLOP/s (against four waves, timed in turn, 195 and 212;
// 206 where all slots gather the same 256 rows: not the fetches); 65536 gathered
// slots of 64 experts by 2048 x 1024, gated, in the 16-bit unit 264 us, 1.04 PFLOP/s
// (eight waves 286).  Zeros take four fifths of that time: the clock falls with the bits
// that change, which is also why fewer copies to LDS count.  In the 16-bit unit a wave
// widens 12 tiles for 32 products (192 conversions at half rate beside 128 matrix
// instructions): the vector unit is as busy as the matrix unit.
#pragma once

#include <type_traits>

#include "eb_expert_product.h"
#include "eb_internal.h"

namespace eb_product {

typedef __amdgpu_buffer_rsrc_t Buffer;

__device__ __forceinline__ Buffer buffer_of(const void *p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, bytes, 0x00020000);
}

// kBytes per lane from a buffer to LDS, lane after lane from `to`.  The whole
// offset is the lane's: a scalar one would be left out of the bounds check, which
// gives zeros for what K's last block has past the last row.
template <int kBytes>
__device__ __forceinline__ void copy_to_lds(Buffer from, void *to, uint32_t offset)
{
    static_assert(kBytes == 16 || kBytes == 4, "");
    const auto lds = (__attribute__((address_space(3))) void *)to;
    if constexpr (kBytes == 16)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lds, 16, offset, 0, 0, 0);
    else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, lds, 4, offset, 0, 0, 0);
}

template <int kTokens16_, int kRows16_, int kAcrossT_, bool kWide_, bool kGate_, bool kFp8_>
struct TileShape {
    static constexpr int kTokens16 = kTokens16_, kRows16 = kRows16_, kAcrossT = kAcrossT_;
    static constexpr bool kWide = kWide_, kGate = kGate_, kFp8 = kFp8_;
    static constexpr bool kOwn = kAcrossT == 1; // a wave's weight rows are its own
    static constexpr int kAcrossR = 4;
    static constexpr int kWaves = kAcrossT * kAcrossR;
    static constexpr int kThreads = kWaves * kWave;
    static constexpr int kHeight = kTokens16 * kAcrossT * 16; // slots
    static constexpr int kLines = kRows16 * kAcrossR * 16;    // weight rows
    static constexpr int kOut16 = kGate ? kRows16 / 2 : kRows16;
    static constexpr int kColumns = kOut16 * kAcrossR * 16;   // outputs
    static constexpr int kCopiesX = kHeight / 8 / kWaves, kCopiesW = kLines / 8 / kWaves; // per wave and block
    static constexpr int kOutBlocks = kColumns / kBlock;
    // Parts in which 16- and 8-bit outputs pass through LDS: that of the weights, or of a stage.
    static constexpr int kOutBytes = kWide && !kFp8 ? 0 : kHeight * kColumns * (kFp8 ? 1 : 2);
    static constexpr int kLdsBytes = (kLines + (kOwn ? 0 : kHeight)) * kBlock;
    static constexpr int kPasses = kOutBytes <= kLdsBytes ? 1 : 2;
    static_assert(kOutBytes <= kPasses * kLdsBytes && kTokens16 % kPasses == 0, "whole passes");
    static_assert(kHeight % (8 * kWaves) == 0 && kLines % (8 * kWaves) == 0, "whole copies");
    static_assert((!kFp8 || kColumns % kBlock == 0) && kBlock % (kOut16 * 16) == 0, "whole blocks of outputs, and a wave's lie in one");
};

struct alignas(16) Chunk {
    char byte[16];
};

// One block of K of the tokens, and of the weights.
template <typename S>
struct TokenBlock {
    Chunk row[S::kHeight][8];
    float scale[S::kHeight > kWave ? S::kHeight : kWave]; // copied by whole waves
};
template <typename S>
struct WeightBlock {
    Chunk row[S::kLines][8];
};
template <typename S>
struct Stage {
    TokenBlock<S> tokens;
    WeightBlock<S> weights;
};

// Workgroups are dealt to the 8 XCDs in turn.  Each takes runs of 32 tiles (its
// compute units), the runs in turn, so that tiles that share operands share an
// L2 and the empty tiles at the end spread over all.
__device__ __forceinline__ uint32_t tile_in_order(uint32_t index, uint32_t count)
{
    constexpr uint32_t kXcds = 8, kRun = 32;
    const uint32_t whole = count / (kXcds * kRun) * (kXcds * kRun);
    if (index >= whole) return index;
    const uint32_t xcd = index % kXcds, nth = index / kXcds;
    return (nth / kRun * kXcds + xcd) * kRun + nth % kRun;
}

constexpr uint32_t kBand = 4; // slot tiles that take their columns together

template <typename S>
__global__ __launch_bounds__(S::kThreads, 2) void eb_product_tile(ProductArgs a)
{
    constexpr int T = S::kTokens16, R = S::kRows16;
    // What is copied to while another part is read is a variable of its own: the
    // compiler then sees that those reads need not wait for the copies.
    __shared__ std::conditional_t<S::kOwn, TokenBlock<S>, Stage<S>> part0, part1;
    __shared__ std::conditional_t<S::kOwn, WeightBlock<S>, Chunk> own;
    auto tokens_of = [](auto &part) -> TokenBlock<S> & {
        if constexpr (S::kOwn) return part;
        else return part.tokens;
    };
    auto weights_of = [&](auto &part) -> WeightBlock<S> & {
        if constexpr (S::kOwn) return own;
        else return part.weights;
    };
    TokenBlock<S> &tokens0 = tokens_of(part0), &tokens1 = tokens_of(part1);
    WeightBlock<S> &weights0 = weights_of(part0), &weights1 = weights_of(part1);
    char *const out_tile = S::kOwn ? (char *)&own : (char *)&part0; // after the last block
    __shared__ int most[S::kFp8 ? S::kOutBlocks * S::kHeight : 1];
    __shared__ int32_t slot_of[S::kHeight]; // of the tile's tokens; -1: not written

    const uint32_t at = tile_in_order(blockIdx.x, gridDim.x);
    // kBand slot tiles by all columns: a run of 32 covers 4 x 8 tiles.
    const uint32_t band = at / (kBand * a.column_tiles), in_band = at % (kBand * a.column_tiles);
    const SlotTile tile = slot_tile<S::kHeight>(a, (int32_t)(band * kBand + in_band % kBand));
    if (tile.expert < 0) return;
    const int32_t column0 = (int32_t)(in_band / kBand) * S::kColumns;

    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int across_r = wave % S::kAcrossR, across_t = wave / S::kAcrossR;
    const int in_row = across_r * S::kOut16 * 16; // this wave's first output of the tile's
    const int32_t column = column0 + in_row;

    // Copies of 8 rows each, a row by 8 lanes.  The weights' first: the tokens'
    // wait for their rows' numbers.  Weight rows past the last one are zeros, or
    // under a gate any; what comes of them is not stored.
    const uint32_t chunk = (lane % 8 ^ lane / 8) * 16;
    const int32_t row_bytes = (a.K + 15) / 16 * 16; // of a buffer's last row; past it reads give zeros
    const Buffer w_buffer = buffer_of(a.w + (int64_t)tile.expert * a.N * a.ldw, (uint32_t)((a.N - 1) * a.ldw + row_bytes));
    const uint32_t w_at = lane / 8 * (uint32_t)a.ldw + chunk;
    auto fill_weights = [&](WeightBlock<S> &weights, int32_t kb) {
#pragma unroll
        for (int i = 0; i < S::kCopiesW; ++i) {
            const int line = (wave * S::kCopiesW + i) * 8;
            // Under a gate the rows that a wave multiplies are those of the gate, then those it gates.
            constexpr int kLinesOf = R * 16;
            const int of = line / kLinesOf * S::kOut16 * 16, at = line % kLinesOf;
            const bool up = S::kGate && at >= kLinesOf / 2;
            const int32_t n = column0 + of + (up ? a.width + at - kLinesOf / 2 : at);
            copy_to_lds<16>(w_buffer, &weights.row[line], w_at + ((uint32_t)n * (uint32_t)a.ldw + (uint32_t)kb * kBlock));
        }
    };
    fill_weights(weights0, 0);

    const int64_t x_first = a.tokens ? 0 : tile.first; // the buffer's first row
    const int64_t x_end = a.tokens ? a.x_rows : tile.end;
    const Buffer x_buffer = buffer_of(a.x + x_first * a.ldx, (uint32_t)((x_end - x_first - 1) * a.ldx + row_bytes));
    auto row_of = [&](int token) { // in the buffer; a slot that is not written takes any
        const int32_t m = tile.first + min(token, tile.end - tile.first - 1);
        if (!a.tokens) return m - tile.first;
        const int32_t row = a.tokens[m];
        return row >= 0 && row < a.x_rows ? row : 0;
    };
    for (int i = threadIdx.x; i < S::kHeight; i += S::kThreads) {
        int32_t slot = i < tile.end - tile.first ? tile.first + i : -1;
        if (a.tokens && slot >= 0 && (a.tokens[slot] < 0 || a.tokens[slot] >= a.x_rows)) slot = -1;
        slot_of[i] = slot;
    }
    uint32_t x_at[S::kCopiesX];
#pragma unroll
    for (int i = 0; i < S::kCopiesX; ++i) x_at[i] = (uint32_t)row_of((wave * S::kCopiesX + i) * 8 + lane / 8) * (uint32_t)a.ldx + chunk;
    // Scales: wave w copies those of slots w * 64 + lane (past the tile: any).
    const bool copies_scales = wave < (S::kHeight + kWave - 1) / kWave;
    const uint32_t scale_at = (uint32_t)row_of(threadIdx.x % S::kHeight) * 4;
    auto fill_tokens = [&](TokenBlock<S> &s, int32_t kb) {
#pragma unroll
        for (int i = 0; i < S::kCopiesX; ++i) copy_to_lds<16>(x_buffer, &s.row[(wave * S::kCopiesX + i) * 8], x_at[i] + (uint32_t)kb * kBlock);
        if (copies_scales)
            copy_to_lds<4>(buffer_of(a.x_scales + kb * a.ldxs + x_first, (uint32_t)(x_end - x_first) * 4), &s.scale[wave * kWave], scale_at);
    };
    fill_tokens(tokens0, 0);
    auto fill = [&](TokenBlock<S> &s, WeightBlock<S> &weights, int32_t kb) {
        fill_tokens(s, kb);
        if constexpr (!S::kOwn) fill_weights(weights, kb);
    };
    // K's last block: what was copied from past a row's end becomes zeros.
    auto cut = [&](TokenBlock<S> &s, WeightBlock<S> &weights, int left) {
        for (int i = threadIdx.x; i < S::kHeight + S::kLines; i += S::kThreads) {
            const int row = i < S::kHeight ? i : i - S::kHeight;
            Chunk *line = i < S::kHeight ? s.row[row] : weights.row[row];
            for (int c = left / 16; c < 8; ++c) {
                i32x4 *p = (i32x4 *)&line[c ^ row % 8];
                *p = first_bytes(*p, left - c * 16);
            }
        }
        __syncthreads();
    };

    const int32_t block = min(column / kBlock, a.row_blocks - 1);
    const float *w_scale = a.w_scales + ((int64_t)tile.expert * a.w_blocks + block) * a.k_blocks;
    const float *w_scale2 = w_scale + (S::kGate ? (int64_t)a.row_blocks * a.k_blocks : 0);

    f32x4 sum[R][T] = {};
    // The weights' scales of a block, loaded when the block before has been read
    // from LDS: with a scalar load among them a wave waits for all its reads.
    float sw_next = eb_detail::scalar_load(w_scale), sw2_next = eb_detail::scalar_load(w_scale2);
    auto multiply = [&](const TokenBlock<S> &s, WeightBlock<S> &weights, int32_t kb) {
        const float sw = sw_next, sw2 = S::kGate ? sw2_next : sw;
        const int p = lane / 16 ^ lane % 8;
        const Chunk(*ws)[8] = &weights.row[across_r * R * 16 + lane % 16], (*xs)[8] = &s.row[across_t * T * 16 + lane % 16];
        const float *scales = &s.scale[across_t * T * 16 + lane % 16];
        auto read = [&](const Chunk(*from)[8], int tile16) {
            return operand(*(const i32x4 *)&from[tile16 * 16][p], *(const i32x4 *)&from[tile16 * 16][p ^ 4]);
        };
        // The sums take a token tile's products while the next tile's are made.
        using Operand = std::conditional_t<S::kWide, Wide, i32x8>;
        auto fit = [](i32x8 v) {
            if constexpr (S::kWide) return widen8(v);
            else return v;
        };
        Operand w[R];
        i32x8 next = read(xs, 0);
        float next_scale = scales[0];
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = fit(read(ws, r));
        if constexpr (S::kOwn) { // all of this wave's weights are read: the next block's may come
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xC07F); // lgkmcnt(0)
            if (kb + 1 < a.k_blocks) fill_weights(weights, kb + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        // Products on their way to the sums: those of the kDelay tiles of 16 x 16
        // (in the order of tokens, then rows) before the one in work.
        constexpr int kDelay = S::kWide ? 1 : R;
        f32x4 product[kDelay];
        float f[2], f2[2]; // factors of even and odd token tiles
        auto add = [&](int i) {
            const int t = i / R, r = i % R;
            const float factor = r < S::kOut16 ? f[t % 2] : f2[t % 2];
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[r][t][j] = fmaf(product[i % kDelay][j], factor, sum[r][t][j]);
            // Here, not where the sums are next read: the compiler would keep every product until then.
            asm volatile("" : "+v"(sum[r][t]));
        };
#pragma unroll
        for (int t = 0; t < T; ++t) {
            if constexpr (!S::kOwn) {
                // The wave that is behind goes first: a SIMD's two then reach the barrier together.
                switch (t * 4 / T) {
                case 0: __builtin_amdgcn_s_setprio(3); break;
                case 1: __builtin_amdgcn_s_setprio(2); break;
                case 2: __builtin_amdgcn_s_setprio(1); break;
                default: __builtin_amdgcn_s_setprio(0);
                }
            }
            const Operand x = fit(next);
            f[t % 2] = next_scale * sw;
            f2[t % 2] = S::kGate ? next_scale * sw2 : f[t % 2];
            if (t + 1 < T) {
                next = read(xs, t + 1);
                next_scale = scales[(t + 1) * 16];
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int i = t * R + r;
                if (i >= kDelay) add(i - kDelay);
                product[i % kDelay] = block_product(w[r], x);
            }
            // The vector instructions evenly between the matrix instructions.
#pragma unroll
            for (int i = 0; i < (S::kWide ? 4 * R : R); ++i) {
                __builtin_amdgcn_sched_group_barrier(0x002, S::kWide ? 2 : 4, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        const int32_t after = min(kb + 1, a.k_blocks - 1);
        sw_next = eb_detail::scalar_load(w_scale + after);
        if constexpr (S::kGate) sw2_next = eb_detail::scalar_load(w_scale2 + after);
#pragma unroll
        for (int i = R * T - kDelay; i < R * T; ++i) add(i);
        __builtin_amdgcn_sched_barrier(0);
    };
    // This block's copies have landed for all waves, and all are done with the
    // block before it.
    auto arrive = [&] {
        __builtin_amdgcn_s_waitcnt(0x0F70); // vmcnt(0)
        __syncthreads();
    };
    const int tail = a.K % kBlock;
    int32_t kb = 0;
    for (; kb + 1 < a.k_blocks; kb += 2) {
        arrive();
        fill(tokens1, weights1, kb + 1);
        multiply(tokens0, weights0, kb);
        arrive();
        if (kb + 2 < a.k_blocks) fill(tokens0, weights0, kb + 2);
        else if (tail) cut(tokens1, weights1, tail);
        multiply(tokens1, weights1, kb + 1);
    }
    if (kb < a.k_blocks) {
        arrive();
        if (tail) cut(tokens0, weights0, tail);
        multiply(tokens0, weights0, kb);
    }

    finish<R, T, S::kGate>(a, tile.expert, column, sum);
    if constexpr (S::kWide && !S::kFp8) {
        // fp32: a lane's four outputs are 16 bytes, four lanes' 64 of a line.  (16-bit
        // outputs of exact sums: half of that.)
        int32_t slot[T];
#pragma unroll
        for (int t = 0; t < T; ++t) slot[t] = slot_of[(across_t * T + t) * 16 + lane % 16];
        store_floats<S::kOut16>(a, column, slot, sum);
        return;
    }
    // Through LDS, so that rows are written in whole lines: token after token of
    // kColumns outputs, chunk c of 16 bytes at place c ^ token % 16 (a wave's 16
    // tokens on all banks).  kPasses parts of the tokens where all do not fit.
    __syncthreads();
    constexpr int kSize = S::kFp8 ? 1 : 2, kChunks = S::kColumns * kSize / 16;
    constexpr int kPasses = S::kPasses;
    auto chunk_of = [&](int token, int c) { return out_tile + (token * kChunks + (c ^ token % (kChunks < 16 ? kChunks : 16))) * 16; };
    auto to_slots = [&](int pass) {
        const int left = min(a.width - column0, S::kColumns) * kSize; // bytes of a row
        for (int i = threadIdx.x; i < S::kHeight / kPasses * kChunks; i += S::kThreads) {
            // Of each kAcrossT-th of the tile's tokens a pass takes T / kPasses tiles of 16.
            constexpr int kPart = T / kPasses * 16;
            const int j = i / kChunks, c = i % kChunks;
            const int32_t m = slot_of[j / kPart * T * 16 + pass * kPart + j % kPart];
            if (c * 16 >= left || m < 0) continue;
            const char *from = chunk_of(j, c);
            char *to = (char *)a.out + ((int64_t)m * a.ldo + column0) * kSize + c * 16;
            if (a.vector_out && c * 16 + 16 <= left) {
                *(i32x4 *)to = *(const i32x4 *)from;
            } else {
                using Element = std::conditional_t<kSize == 2, int16_t, char>;
                const int n = min(16, left - c * 16) / kSize;
                for (int k = 0; k < n; ++k) ((Element *)to)[k] = ((const Element *)from)[k];
            }
        }
    };
    const int part = lane / 16 * 4;
    if constexpr (S::kFp8) {
        int *mine = &most[in_row / kBlock * S::kHeight + across_t * T * 16];
        for (int i = threadIdx.x; i < S::kOutBlocks * S::kHeight; i += S::kThreads) most[i] = 0;
        __syncthreads();
        if (column + S::kOut16 * 16 > a.width) { // outputs past the width do not count
#pragma unroll
            for (int r = 0; r < S::kOut16; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int t = 0; t < T; ++t) sum[r][t][i] = column + r * 16 + part + i < a.width ? sum[r][t][i] : 0.f;
        }
        most_of_outputs<S::kOut16>(sum, mine);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int token = (across_t * T + t) * 16 + lane % 16;
            const float f = block_scale(mine[t * 16 + lane % 16]);
#pragma unroll
            for (int r = 0; r < S::kOut16; ++r)
                *(int *)(chunk_of(token, in_row / 16 + r) + part) = pack_fp8(sum[r][t], f);
        }
        __syncthreads();
        to_slots(0);
        for (int i = threadIdx.x; i < S::kOutBlocks * S::kHeight; i += S::kThreads) {
            const int32_t m = slot_of[i % S::kHeight], b = column0 / kBlock + i / S::kHeight;
            if (m < 0 || b >= a.row_blocks) continue;
            a.out_scales[(int64_t)b * a.ldos + m] = block_scale(most[i]);
        }
    } else {
#pragma unroll
        for (int pass = 0; pass < kPasses; ++pass) {
            if (pass > 0) __syncthreads();
            auto to_lds = [&](auto bits) {
#pragma unroll
                for (int u = 0; u < T / kPasses; ++u) {
                    const int t = pass * (T / kPasses) + u, token = (across_t * (T / kPasses) + u) * 16 + lane % 16;
#pragma unroll
                    for (int r = 0; r < S::kOut16; ++r) {
                        const int c = in_row + r * 16 + part;
                        *(uint2 *)(chunk_of(token, c / 8) + c % 8 * 2) = bits(sum[r][t]);
                    }
                }
            };
            if (a.out_type == EB_F16) to_lds([](f32x4 v) { return pack16<_Float16>(v); });
            else to_lds([](f32x4 v) { return pack16<__bf16>(v); });
            __syncthreads();
            to_slots(pass);
        }
    }
}

template <typename S>
KernelPlan tile_plan()
{
    return {eb_product_tile<S>, S::kHeight, S::kColumns, S::kThreads, kBand};
}

} // namespace eb_product
