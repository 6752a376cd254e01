// eb_expert_product for few slots of few experts: bound by latency and by the
// weights' way to the few compute units that have them (one slot by 2048 x 1024 3.4
// us; 64 by 2048 x 4096 10.7).  And for operands beyond 32-bit offsets: all
// addresses here have 64 bits.
//
// A workgroup of eight waves takes up to 16 slots of an expert and a run of its
// weight rows: kAcross waves side by side, each with kRows tiles of 16 rows, and
// kWaves / kAcross waves along K with every such block of 128 each, joined in LDS
// in a fixed order.  Where the outputs are not quantised that is 16 rows (with a
// gate, 16 of each half) and all waves along K: many workgroups with short ways.
// The products are taken in the 16-bit unit, exact: its rate does not matter
// here.  Both operands come straight from global memory into the registers of
// the matrix instructions; each weight is read once per 16 slots, and a wave's
// 16 rows of 128 bytes are whole lines.

#include "eb_expert_product.h"

namespace eb_product {

namespace {

constexpr int kWaves = 8;
constexpr int kHeight = 16; // slots of a workgroup

template <int kRows, int kAcross, bool kGate, bool kFp8>
__global__ __launch_bounds__(kWaves *kWave) void eb_product_stream(ProductArgs a)
{
    constexpr int kAlong = kWaves / kAcross; // waves along K
    constexpr int kOut = kGate ? kRows / 2 : kRows;
    constexpr int kColumns = kAcross * kOut * 16;
    static_assert(!kFp8 || kColumns == kBlock, "a scale needs its whole block in the workgroup");
    __shared__ f32x4 part_of[kAlong > 1 ? (kAlong - 1) * kAcross * kRows * kWave : 1];
    __shared__ int most[kFp8 ? kHeight : 1];

    const SlotTile tile = slot_tile<kHeight>(a, blockIdx.x / a.column_tiles);
    if (tile.expert < 0) return;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int across = wave % kAcross, along = wave / kAcross;
    const int32_t column = (blockIdx.x % a.column_tiles) * kColumns + across * kOut * 16;
    const int chunk = lane / 16;

    const char *wrow[kRows];
    const float *wscale[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const bool up = kGate && r >= kOut;
        const int32_t c = column + (up ? r - kOut : r) * 16;
        const int64_t n = (up ? a.width : 0) + min(c + lane % 16, a.width - 1);
        wrow[r] = a.w + ((int64_t)tile.expert * a.N + n) * a.ldw;
        const int32_t b = min(c / kBlock, a.row_blocks - 1) + (up ? a.row_blocks : 0);
        wscale[r] = a.w_scales + ((int64_t)tile.expert * a.w_blocks + b) * a.k_blocks;
    }
    const int32_t m = tile.first + min(lane % 16, tile.end - tile.first - 1);
    const int32_t row = a.tokens ? a.tokens[m] : m;
    const bool fits = row >= 0 && row < a.x_rows;
    const int32_t slot[1] = {lane % 16 < tile.end - tile.first && fits ? m : -1};
    const char *const xrow = a.x + (fits ? row : 0) * a.ldx;
    const float *const xscale = a.x_scales + (fits ? row : 0);
    f32x4 sum[kRows][1] = {};
    if (a.x_rows > 0) {
        for (int32_t kb = along; kb < a.k_blocks; kb += kAlong) {
            const int32_t k0 = kb * kBlock;
            const int left = a.K - k0; // bytes of this block
            // A chunk past the end is read at the block's start and cleared.
            const int lo = chunk * 16 < left ? chunk * 16 : 0, hi = chunk * 16 + 64 < left ? chunk * 16 + 64 : 0;
            i32x8 w[kRows];
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                w[r] = operand(*(const i32x4 *)(wrow[r] + k0 + lo), *(const i32x4 *)(wrow[r] + k0 + hi));
            i32x8 x = operand(*(const i32x4 *)(xrow + k0 + lo), *(const i32x4 *)(xrow + k0 + hi));
            const float sx = xscale[kb * a.ldxs];
            if (left < kBlock) {
#pragma unroll
                for (int r = 0; r < kRows; ++r)
                    w[r] = operand(first_bytes(w[r].lo, left - chunk * 16), first_bytes(w[r].hi, left - chunk * 16 - 64));
                x = operand(first_bytes(x.lo, left - chunk * 16), first_bytes(x.hi, left - chunk * 16 - 64));
            }
            const Wide wide_x = widen8(x);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const f32x4 p = block_product(widen8(w[r]), wide_x);
                const float f = sx * wscale[r][kb];
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[r][0][i] = fmaf(p[i], f, sum[r][0][i]);
            }
        }
    }
    if constexpr (kAlong > 1) {
        auto place = [&](int w, int r) { return ((w - 1) * kAcross + across) * kRows + r; };
        if (along > 0) {
#pragma unroll
            for (int r = 0; r < kRows; ++r) part_of[place(along, r) * kWave + lane] = sum[r][0];
        }
        __syncthreads();
        if (along == 0) {
            for (int w = 1; w < kAlong; ++w)
#pragma unroll
                for (int r = 0; r < kRows; ++r) sum[r][0] += part_of[place(w, r) * kWave + lane];
        }
    }
    if (along == 0) finish<kRows, 1, kGate>(a, tile.expert, column, sum);
    if constexpr (kFp8) {
        if (threadIdx.x < kHeight) most[threadIdx.x] = 0;
        __syncthreads();
        if (along == 0) most_of_outputs<kOut>(sum, most);
        __syncthreads();
        if (along == 0) store_fp8<kOut>(a, column, slot, sum, most, across == 0);
    } else {
        if (along == 0) store_floats<kOut>(a, column, slot, sum);
    }
}

template <int kRows, int kAcross, bool kGate, bool kFp8>
KernelPlan plan()
{
    return {eb_product_stream<kRows, kAcross, kGate, kFp8>, kHeight, kAcross * (kGate ? kRows / 2 : kRows) * 16, kWaves * kWave, 1};
}

} // namespace

KernelPlan stream_kernel(bool gate, bool fp8)
{
    if (gate) return fp8 ? plan<2, 8, true, true>() : plan<2, 1, true, false>();
    return fp8 ? plan<2, 4, false, true>() : plan<1, 1, false, false>();
}

} // namespace eb_product
