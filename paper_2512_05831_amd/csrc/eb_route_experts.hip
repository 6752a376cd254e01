// Routing to experts: eb_route_experts (include/eb_experts.h).
//
// For token n with router outputs x (E of them):
//   s_e = softmax(x)_e or 1 / (1 + exp(-x_e)),  c_e = s_e + bias_e (or x_e,
//   which orders the same), the K largest c_e of the best groups, w = s there.
// Then a stable counting sort of the N * K pairs by expert.
//
// choose  L = 16 lanes (64 for many experts) hold a token's E values in
//         registers, V each, as integers that order like the floats (an
//         integer maximum takes its other operand straight from another lane).
//         With 16 lanes and 2 < K <= 8: the K-th largest of the lanes' maxima
//         bounds the K best values from below, those above it (eleven or so
//         where K is 8) go to LDS, a lane takes one each and counts the better
//         ones: about 220 instructions, where K rounds of "largest value left,
//         lowest expert that has it, out with it" are 680 (16 values a lane).
//         (Two each where 17 to 32 reach the bound: one token in 25, but then its
//         whole wave.)  Those rounds are taken where more do, and for other K
//         and L.  16384 tokens in all: 8 of 256 experts 17.8 us, by rounds 20.9; 6
//         of 64 13.0 and 13.9; 2 of 128 14.0 and 13.6.  Each workgroup counts its
//         pairs per expert.
// scan    exclusive prefix of each expert's counts over the chunks of kTokens
//         tokens.
// place   each workgroup ranks its pairs within their experts (in pair order:
//         the lanes of a wave that hold the same expert find each other by
//         ballots over the expert's bits) and writes them.
// Choose is bound by vector instructions: 16384 tokens of 256 experts with sigmoid,
// bias and pairs of groups 16 us (0.82 issued a cycle) for 16.8 MB that a copy would
// read in 4; scan and place are 4.5 and 5 us of latency there.
// A launch costs more than the work of a small batch (2.4 us of the caller's time):
// up to 16 tokens, or 128 of at most 64 experts, one workgroup does all of it (us
// a call among others: 64 tokens, 6 of 64 experts 11.4, two launches 13.7; on the GPU
// 6.8 and 7.2; but 64 tokens, 8 of 256 22.5 and 13.8).  Up to kFewPairs pairs there is
// no scan: each workgroup that places kPart pairs counts all of them (8000 pairs of
// 64 experts 13.7, three launches 17.6, on the GPU 10.8 and 11.3; 16000 pairs 13.9 and
// 17.6, on the GPU 13.5 and 11.5: there it is the caller's time that is bought).

#include <hip/hip_runtime.h>

#include <stdint.h>

#include <algorithm>
#include <limits>

#include "../../include/eb.h"
#include "../../include/eb_experts.h"
#include "eb_experts.h"
#include "eb_internal.h"

namespace {

using namespace eb_experts;
using eb_detail::fail;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kChooseThreads = 512; // 32 tokens of 16 lanes
constexpr int kTokens = 32;        // tokens of a chunk
constexpr int kFewWaves = 16;      // of the workgroup that does all
constexpr int kFewTokens = 128, kFewPairs = 16384, kFewExperts = 512;
constexpr int kMostFewPairs = kFewWaves * 64;
constexpr int kFilterTop = 8;      // most experts per token for the filter
constexpr int kMostExperts = 1024;
constexpr int kMostTop = 64;
constexpr int kMostGroups = 32;

constexpr int kNoneKey = (int)0x807FFFFF; // the key of -infinity
constexpr float kInf = __builtin_inff();

struct RouteArgs {
    const void *scores;
    const float *bias;
    int64_t ld;
    int64_t N;
    int32_t E, K;
    int32_t sigmoid, renormalize, pair;
    int32_t groups, top_groups, group_size;
    uint32_t group_magic; // e / group_size == e * group_magic >> 20 for e < 1024
    float scale;
    int32_t lo, held; // this GPU's experts [lo, lo + held)
    int32_t *ids;
    float *weights;
    int32_t *offsets, *tokens, *slots;
    int32_t each;     // tokens of a workgroup of choose
    uint32_t *counts; // [held][chunks + 1], the total last, or NULL: none are taken
    int64_t chunks;
};

// An integer that orders like the float (no NaNs; both zeros are equal).
__device__ __forceinline__ int order_key(float v)
{
    const int b = __float_as_int(v + 0.f);
    return b ^ ((b >> 31) & 0x7FFFFFFF);
}

__device__ __forceinline__ float key_value(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)); }

// Rounded as torch's 1 / (1 + exp(-x)) is: choices rest on its last bit.
__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

// exp(v) of v <= 0 within 2 ulp: 2^h (1 + l ln 2), h + l = v log2(e).
__device__ __forceinline__ float exp_of(float v)
{
    const float h = v * 1.44269502f, l = fmaf(v, 1.44269502f, -h) + v * 1.92596303e-8f, e = __builtin_amdgcn_exp2f(h);
    return h > -126.f ? fmaf(e, l * 0.693147181f, e) : 0.f;
}

// A key and its expert as one integer: of equal keys the lower expert is larger.
__device__ __forceinline__ int64_t candidate(int key, int expert) { return (int64_t)key << 32 | (0x7FFFFFFF - expert); }

// What a lane group has in LDS for one token.
template <int L, int V>
struct TokenSpace {
    union {
        struct {
            float judged[L * V + kMostGroups]; // scores, a word of padding per group
            int group_key[kMostGroups];
        };
        struct {
            int64_t found[32 + L]; // from 32 on: what is not wanted
            int64_t best[kFilterTop];
        };
    };
};

// The K best of a token's experts, of which lane k gets the k-th: its expert
// (-1: none left) and key.  key[v] of lane i is expert v * L + i's.
template <int L, int V>
__device__ __forceinline__ void best_by_rounds(int (&key)[V], int lane, int K, int &id, int &id_key)
{
    for (int k = 0; k < K; ++k) {
        int m = key[0];
#pragma unroll
        for (int v = 1; v < V; ++v) m = max(m, key[v]);
        m = max_lanes<L>(m);
        if (m == kNoneKey) break; // the same for all lanes of a group
        int e = 0x7FFFFFFF;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) e = key[v] == m ? v * L + lane : e;
        e = min_lanes<L>(e);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = e == v * L + lane ? kNoneKey : key[v];
        if (lane == k) {
            id = e;
            id_key = m;
        }
    }
}

template <int V>
__device__ __forceinline__ void best_by_filter(int (&key)[V], int lane, int K, TokenSpace<16, V> &space, int &id, int &id_key)
{
    int m = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = max(m, key[v]);
    int greater = 0;
#define EB_COUNT(S) greater += rotate16<S>(m) > m;
    EB_COUNT(1) EB_COUNT(2) EB_COUNT(3) EB_COUNT(4) EB_COUNT(5) EB_COUNT(6) EB_COUNT(7) EB_COUNT(8)
    EB_COUNT(9) EB_COUNT(10) EB_COUNT(11) EB_COUNT(12) EB_COUNT(13) EB_COUNT(14) EB_COUNT(15)
#undef EB_COUNT
    const int bound = max(min_lanes<16>(greater < K ? m : 0x7FFFFFFF), kNoneKey + 1);
    int mine = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) mine += key[v] >= bound;
    int upto = mine; // inclusive prefix over the 16 lanes
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x111, 0xF, 0xF, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x112, 0xF, 0xF, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x114, 0xF, 0xF, false);
    upto += __builtin_amdgcn_update_dpp(0, upto, 0x118, 0xF, 0xF, false);
    const int n = max_lanes<16>(upto);
    if (__any(n > 32)) return best_by_rounds<16, V>(key, lane, K, id, id_key);
    const bool second = __any(n > 16); // a lane then takes two
    const int64_t none = candidate(kNoneKey, 0x7FFFFFFF);
    space.found[lane] = none;
    space.found[16 + lane] = none;
    wave_fence();
    int at = upto - mine;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const bool wanted = key[v] >= bound;
        space.found[wanted ? at : 32 + lane] = candidate(key[v], v * 16 + lane);
        at += wanted;
    }
    wave_fence();
    auto settle = [&](int64_t own) {
        int rank = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) rank += space.found[j] > own;
        if (second) {
#pragma unroll
            for (int j = 16; j < 32; ++j) rank += space.found[j] > own;
        }
        if (own != none && rank < kFilterTop) space.best[rank] = own;
    };
    settle(space.found[lane]);
    if (second) settle(space.found[16 + lane]);
    wave_fence();
    if (lane < min(n, K)) {
        const int64_t c = space.best[lane];
        id = 0x7FFFFFFF - (int)c;
        id_key = (int)(c >> 32);
    }
    wave_fence(); // the next token's values come to the same LDS
}

// One token by a lane group: lane k < K returns its k-th expert and weight.
template <int L, int V, typename T>
__device__ __forceinline__ void choose(const RouteArgs &a, int64_t n, int lane, TokenSpace<L, V> &space, int &id, float &weight)
{
    const T *row = (const T *)a.scores + n * a.ld;
    float x[V];
    int key[V];
    const bool scored = a.bias || a.pair; // the choice needs the scores themselves
    T raw[V];
    float bias[V];
#pragma unroll
    for (int v = 0; v < V; ++v) raw[v] = row[min(v * L + lane, a.E - 1)];
    if (a.bias) {
#pragma unroll
        for (int v = 0; v < V; ++v) bias[v] = a.bias[min(v * L + lane, a.E - 1)];
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = v * L + lane;
        float f = e < a.E ? widen(raw[v]) : -kInf;
        f = f == f ? f : -kInf;
        x[v] = f < kInf ? f : __FLT_MAX__;
        key[v] = order_key(x[v]);
    }
    float top_x = 0.f, total = 1.f;
    if (!a.sigmoid) {
        int most = key[0];
#pragma unroll
        for (int v = 1; v < V; ++v) most = max(most, key[v]);
        top_x = key_value(max_lanes<L>(most));
        if (scored || !a.renormalize) {
            float t = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) t += x[v] > -kInf ? exp_of(x[v] - top_x) : 0.f;
            total = sum_lanes<L>(t);
        }
    }
    if (scored) {
        // A branch around each loop, not in it: the values' chains then overlap.
        float s[V];
        if (a.sigmoid) {
#pragma unroll
            for (int v = 0; v < V; ++v) s[v] = sigmoid(x[v]);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) s[v] = exp_of(x[v] - top_x) / total;
        }
        if (a.bias) {
#pragma unroll
            for (int v = 0; v < V; ++v) s[v] += bias[v];
        }
        // A NaN bias makes its expert unfit, as a NaN score does.
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = x[v] > -kInf && s[v] == s[v] ? s[v] : -kInf;
        if (a.pair) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int e = v * L + lane;
                space.judged[min((int)(e + (e * a.group_magic >> 20)), L * V + kMostGroups - 1)] = s[v];
            }
        }
        if (a.bias) {
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = order_key(s[v]);
        }
    }
    if (a.groups > 1) {
        if (!a.pair) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int e = v * L + lane;
                space.judged[min((int)(e + (e * a.group_magic >> 20)), L * V + kMostGroups - 1)] = key_value(key[v]);
            }
        }
        wave_fence();
        for (int g = lane; g < a.groups; g += L) {
            float best = -kInf, next = -kInf;
#pragma unroll 8
            for (int i = 0; i < a.group_size; ++i) {
                const float s = space.judged[g * (a.group_size + 1) + i];
                next = fmaxf(next, fminf(best, s));
                best = fmaxf(best, s);
            }
            space.group_key[g] = order_key(!a.pair ? best : next > -kInf ? best + next : -kInf);
        }
        wave_fence();
        int kept = 0;
        for (int g = lane; g < a.groups; g += L) {
            const int k = space.group_key[g];
            int better = 0;
#pragma unroll 8
            for (int h = 0; h < a.groups; ++h) {
                const int o = space.group_key[h];
                better += o > k || (o == k && h < g);
            }
            kept |= better < a.top_groups ? 1 << g : 0;
        }
        kept = or_lanes<L>(kept);
        wave_fence();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const uint32_t e = v * L + lane;
            if (!(kept >> ((e * a.group_magic >> 20) & 31) & 1)) key[v] = kNoneKey;
        }
    }
    int id_key = kNoneKey;
    id = -1;
    if constexpr (L == 16 && V >= 4) {
        if (a.K > 2 && a.K <= kFilterTop) best_by_filter<V>(key, lane, a.K, space, id, id_key);
        else best_by_rounds<L, V>(key, lane, a.K, id, id_key);
    } else {
        best_by_rounds<L, V>(key, lane, a.K, id, id_key);
    }
    // The key is x's, or the biased score's: then x is read again.
    float x_of = id < 0 ? -kInf : key_value(id_key);
    if (a.bias && id >= 0) {
        x_of = widen(row[id]);
        x_of = x_of < kInf ? x_of : __FLT_MAX__;
    }
    float w = id < 0 ? 0.f : a.sigmoid ? sigmoid(x_of) : exp_of(x_of - top_x);
    if (a.renormalize) {
        if (!a.sigmoid && scored) { // against the largest of the chosen: they may lie far below top_x
            const float m = key_value(max_lanes<L>(order_key(x_of)));
            w = id < 0 ? 0.f : exp_of(x_of - m);
        }
        if (a.sigmoid) { // e^-m / (1 + e^-x): no underflow where all x are low
            const float m = fminf(key_value(max_lanes<L>(order_key(x_of))), 0.f);
            w = id < 0 ? 0.f : 1.f / (expf(m) + expf(m - x_of));
        }
        const float t = sum_lanes<L>(w);
        w = t > 0.f ? w / t : 0.f;
    } else if (!a.sigmoid) {
        w = id < 0 ? 0.f : w / total;
    }
    weight = id < 0 ? 0.f : w * a.scale; // the scale may be infinite or NaN
}

// The pair's expert as one of this GPU's, or -1.
__device__ __forceinline__ int held_expert(const RouteArgs &a, int id)
{
    return id >= a.lo && id - a.lo < a.held ? id - a.lo : -1;
}

template <int L, int V, typename T>
__global__ __launch_bounds__(kChooseThreads, L *V <= 512 ? 4 : 2) void eb_route_choose(RouteArgs a)
{
    constexpr int kPass = kChooseThreads / L; // tokens a workgroup takes at a time
    __shared__ uint32_t count[kMostExperts];
    __shared__ TokenSpace<L, V> space[kPass];

    const int lane = threadIdx.x % L, mine = threadIdx.x / L; // token of a pass
    if (a.counts) {
        for (int j = threadIdx.x; j < a.held; j += kChooseThreads) count[j] = 0;
        __syncthreads();
    }
    const int each = kPass >= kTokens ? kTokens : a.each;
    for (int p = 0; p < each; p += kPass) {
        const int64_t n = (int64_t)blockIdx.x * each + p + mine;
        if (n >= a.N) break; // ends for whole lane groups; no barrier in the loop
        int id;
        float w;
        choose<L, V, T>(a, n, lane, space[mine], id, w);
        if (lane < a.K) {
            a.ids[n * a.K + lane] = id;
            a.weights[n * a.K + lane] = w;
            if (a.counts && held_expert(a, id) >= 0) atomicAdd(&count[id - a.lo], 1u);
        }
    }
    if (!a.counts) return;
    __syncthreads();
    for (int j = threadIdx.x; j < a.held; j += kChooseThreads) a.counts[j * (a.chunks + 1) + blockIdx.x] = count[j];
}

// The lanes of a wave that hold the same expert j (those with j < 0: none).
__device__ __forceinline__ uint64_t same_expert(int j, int bits)
{
    uint64_t same = __ballot(j >= 0);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(j >> b & 1);
        same &= j >> b & 1 ? set : ~set;
    }
    return same;
}

// Inclusive prefix over a wave.
__device__ __forceinline__ uint32_t prefix_in_wave(uint32_t v)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const uint32_t o = __shfl_up(v, d);
        v += (int)(threadIdx.x % kWave) >= d ? o : 0;
    }
    return v;
}

// Scan and placing of the pairs [begin, end) by a workgroup of kFewWaves waves,
// which counts all the others too.  expert_of(p): the held expert of pair p, or -1.
constexpr int kAllThreads = kFewWaves * kWave;

struct PlaceSpace {
    uint32_t next[kFewWaves][kMostExperts]; // counts, then the next slot, per wave and expert
    uint32_t before[kMostExperts], after[kMostExperts]; // pairs of other workgroups
};

template <typename ExpertOf>
__device__ __forceinline__ void place_all(const RouteArgs &a, PlaceSpace &space, uint32_t (&wave_sum)[kFewWaves], int begin, int end,
                                          ExpertOf expert_of)
{
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    // A wave takes a run of the pairs.
    const int pairs = (int)a.N * a.K, run = (end - begin + kFewWaves - 1) / kFewWaves;
    const int p0 = min(end, begin + wave * run), p1 = min(end, p0 + run);
    const int bits = 32 - __clz(a.held | 1);
    for (int j = lane; j < a.held; j += kWave) space.next[wave][j] = 0;
    for (int j = threadIdx.x; j < a.held; j += kAllThreads) space.before[j] = space.after[j] = 0;
    wave_fence();
    for (int p = p0 + lane; p < p1; p += kWave) {
        const int j = expert_of(p);
        if (j >= 0) atomicAdd(&space.next[wave][j], 1u);
    }
    __syncthreads();
    auto count = [&](int from, int to, uint32_t *counts) {
        constexpr int kEach = 8; // loads under way
        for (int q = from; q < to; q += kEach * kAllThreads) {
            int e[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int p = q + i * kAllThreads + (int)threadIdx.x;
                e[i] = p < to ? expert_of(p) : -1;
            }
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (q + i * kAllThreads >= to) break;
                const int lead = __builtin_amdgcn_readfirstlane(e[i]);
                if (__all(e[i] == lead)) {
                    if (lead >= 0 && lane == 0) atomicAdd(&counts[lead], (uint32_t)kWave);
                } else if (a.held > 8) {
                    if (e[i] >= 0) atomicAdd(&counts[e[i]], 1u);
                } else { // many lanes at one address: one for all of them
                    const uint64_t same = same_expert(e[i], bits);
                    if (e[i] >= 0 && (same & ((1ull << lane) - 1)) == 0) atomicAdd(&counts[e[i]], (uint32_t)__popcll(same));
                }
            }
        }
    };
    count(0, begin, space.before);
    count(end, pairs, space.after);
    __syncthreads();
    static_assert(kAllThreads >= kMostExperts, "a thread per expert");
    const int j = threadIdx.x;
    uint32_t mine = 0, sum = 0, earlier = 0;
    if (j < a.held) {
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
            const uint32_t n = space.next[w][j];
            space.next[w][j] = mine;
            mine += n;
        }
        earlier = space.before[j];
        sum = earlier + mine + space.after[j];
    }
    const uint32_t upto = prefix_in_wave(sum);
    if (lane == kWave - 1) wave_sum[wave] = upto;
    __syncthreads();
    uint32_t first = upto - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
        first += w < wave ? wave_sum[w] : 0;
        total += wave_sum[w];
    }
    if (j < a.held) {
        if (begin == 0) a.offsets[j] = (int32_t)first;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) space.next[w][j] += first + earlier;
    }
    if (begin == 0 && j == 0) a.offsets[a.held] = (int32_t)total;
    __syncthreads();
    for (int q = p0; q < p1; q += kWave) {
        const int p = q + lane;
        const int e = p < p1 ? expert_of(p) : -1;
        const uint64_t same = same_expert(e, bits);
        const int rank = __popcll(same & ((1ull << lane) - 1));
        uint32_t at = 0;
        if (e >= 0) at = space.next[wave][e] + rank;
        wave_fence();
        if (e >= 0 && rank == 0) space.next[wave][e] += __popcll(same);
        wave_fence();
        if (p < p1) a.slots[p] = e >= 0 ? (int32_t)at : -1;
        if (e >= 0) a.tokens[at] = p / a.K;
        if (p < p1 && p >= (int)total) a.tokens[p] = -1; // past the last slot
    }
}

// The whole of it for few tokens, in one workgroup.
template <int L, int V, typename T>
__global__ __launch_bounds__(kAllThreads) void eb_route_few(RouteArgs a)
{
    constexpr int kPass = kAllThreads / L;
    __shared__ union {
        TokenSpace<L, V> token[kPass];
        PlaceSpace place;
    } space;
    __shared__ int16_t expert_of[kMostFewPairs];
    __shared__ uint32_t wave_sum[kFewWaves];

    const int lane = threadIdx.x % L;
    for (int p = threadIdx.x / L; p < a.N; p += kPass) {
        int id;
        float w;
        choose<L, V, T>(a, p, lane, space.token[threadIdx.x / L], id, w);
        if (lane < a.K) {
            a.ids[p * a.K + lane] = id;
            a.weights[p * a.K + lane] = w;
            expert_of[p * a.K + lane] = (int16_t)held_expert(a, id);
        }
    }
    if (!a.offsets) return;
    __syncthreads();
    place_all(a, space.place, wave_sum, 0, (int)a.N * a.K, [&](int p) { return (int)expert_of[p]; });
}

constexpr int kPart = 1024; // pairs that a workgroup of it places

__global__ __launch_bounds__(kAllThreads) void eb_route_place_few(RouteArgs a)
{
    __shared__ PlaceSpace space;
    __shared__ uint32_t wave_sum[kFewWaves];
    const int begin = (int)blockIdx.x * kPart;
    place_all(a, space, wave_sum, begin, min((int)a.N * a.K, begin + kPart), [&](int p) { return held_expert(a, a.ids[p]); });
}

// counts[j][c] becomes the pairs of expert j in the chunks before c, the total
// last: a wave per expert.
__global__ __launch_bounds__(kThreads) void eb_route_scan(RouteArgs a)
{
    const int lane = threadIdx.x % kWave;
    const int j = blockIdx.x * kWaves + threadIdx.x / kWave;
    if (j >= a.held) return;
    uint32_t *row = a.counts + j * (a.chunks + 1);
    uint32_t before = 0;
    constexpr int kEach = 8; // loads under way
    for (int64_t c0 = 0; c0 < a.chunks; c0 += kEach * kWave) {
        uint32_t n[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int64_t c = c0 + i * kWave + lane;
            n[i] = c < a.chunks ? row[c] : 0;
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int64_t c = c0 + i * kWave + lane;
            const uint32_t upto = prefix_in_wave(n[i]);
            if (c < a.chunks) row[c] = before + upto - n[i];
            before += __shfl(upto, kWave - 1);
        }
    }
    if (lane == 0) row[a.chunks] = before;
}

__global__ __launch_bounds__(kThreads) void eb_route_place(RouteArgs a)
{
    __shared__ uint32_t next[kWaves][kMostExperts]; // counts, then the next slot, per wave and expert
    __shared__ uint32_t wave_sum[kWaves];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t n0 = (int64_t)blockIdx.x * kTokens;
    const int64_t pairs = a.N * a.K;
    // This wave's pairs: a quarter of the chunk's tokens.
    constexpr int kMine = kTokens / kWaves;
    const int64_t p0 = min(pairs, (n0 + wave * kMine) * a.K), p1 = min(pairs, p0 + (int64_t)kMine * a.K);
    for (int j = lane; j < a.held; j += kWave) next[wave][j] = 0;
    wave_fence();
    for (int64_t p = p0 + lane; p < p1; p += kWave) {
        const int j = held_expert(a, a.ids[p]);
        if (j >= 0) atomicAdd(&next[wave][j], 1u);
    }
    __syncthreads();
    // Slots of the experts before mine: an exclusive prefix over the totals,
    // kThreads experts at a time.
    uint32_t base = 0;
    for (int j0 = 0; j0 < a.held; j0 += kThreads) {
        const int j = j0 + threadIdx.x;
        const uint32_t *row = a.counts + j * (a.chunks + 1);
        const uint32_t mine = j < a.held ? row[a.chunks] : 0;
        const uint32_t sum = prefix_in_wave(mine);
        if (lane == kWave - 1) wave_sum[wave] = sum;
        __syncthreads();
        uint32_t before = base + sum - mine;
        for (int w = 0; w < wave; ++w) before += wave_sum[w];
        for (int w = 0; w < kWaves; ++w) base += wave_sum[w];
        if (j < a.held) {
            if (blockIdx.x == 0) a.offsets[j] = (int32_t)before;
            uint32_t at = before + row[blockIdx.x];
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t n = next[w][j];
                next[w][j] = at;
                at += n;
            }
        }
        __syncthreads();
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[a.held] = (int32_t)base;
    const int bits = 32 - __clz(a.held | 1);
    for (int64_t q = p0; q < p1; q += kWave) {
        const int64_t p = q + lane;
        const int j = p < p1 ? held_expert(a, a.ids[p]) : -1;
        const uint64_t same = same_expert(j, bits);
        const int rank = __popcll(same & ((1ull << lane) - 1));
        uint32_t at = 0;
        if (j >= 0) at = next[wave][j] + rank;
        wave_fence();
        if (j >= 0 && rank == 0) next[wave][j] += __popcll(same);
        wave_fence();
        if (p < p1) a.slots[p] = j >= 0 ? (int32_t)at : -1;
        if (j >= 0) a.tokens[at] = (int32_t)(p / a.K);
        if (p < p1 && p >= base) a.tokens[p] = -1; // past the last slot
    }
}

__global__ void eb_route_none(int32_t *offsets, int32_t n)
{
    for (int j = threadIdx.x; j < n; j += blockDim.x) offsets[j] = 0;
}

// Whether one workgroup does it all: a token per wave, or four where 16 lanes hold
// the experts in four registers each (for more the 16 waves have too few).
bool is_few(int64_t N, int32_t E, int32_t K)
{
    return N <= kFewWaves ? E <= kFewExperts : N <= kFewTokens && N * K <= kMostFewPairs && E <= 64 && K <= 16;
}

template <typename T>
void *few_kernel(int64_t N, int32_t E, int32_t K)
{
    if (N > 4 && E <= 64 && K <= 16) return (void *)eb_route_few<16, 4, T>;
    if (E <= 64) return (void *)eb_route_few<64, 1, T>;
    if (E <= 128) return (void *)eb_route_few<64, 2, T>;
    if (E <= 256) return (void *)eb_route_few<64, 4, T>;
    return (void *)eb_route_few<64, 8, T>;
}

int choose_lanes(int32_t E, int32_t K) { return K <= 16 && E <= 256 ? 16 : 64; }

template <typename T>
void *choose_kernel(bool few, int64_t N, int32_t E, int32_t K)
{
    if (few) return few_kernel<T>(N, E, K);
    if (choose_lanes(E, K) == 16) {
        if (E <= 32) return (void *)eb_route_choose<16, 2, T>;
        if (E <= 64) return (void *)eb_route_choose<16, 4, T>;
        if (E <= 128) return (void *)eb_route_choose<16, 8, T>;
        return (void *)eb_route_choose<16, 16, T>;
    }
    if (E <= 256) return (void *)eb_route_choose<64, 4, T>;
    if (E <= 512) return (void *)eb_route_choose<64, 8, T>;
    return (void *)eb_route_choose<64, 16, T>;
}

int64_t chunks_of(int64_t N) { return (N + kTokens - 1) / kTokens; }

size_t workspace_of(int64_t N, int32_t K, int32_t held)
{
    return N * K <= kFewPairs ? 0 : (size_t)(chunks_of(N) + 1) * (size_t)std::max(held, 1) * 4;
}

int route_impl(const char *who, int64_t N, int32_t E, int32_t K, const void *scores, int32_t dtype, int64_t ld,
               const float *bias, int32_t mode, int32_t groups, int32_t top_groups, float scale, int32_t shard_lo,
               int32_t shard_hi, int32_t *ids, float *weights, int32_t *offsets, int32_t *tokens, int32_t *slots,
               void *workspace, size_t workspace_bytes, void *stream)
{
    if (N < 0 || E < 1 || K < 1 || K > E) return fail(EB_ERR_INVALID, "%s: needs N >= 0 and 1 <= K <= E", who);
    if (dtype != EB_F32 && dtype != EB_F16 && dtype != EB_BF16) return fail(EB_ERR_INVALID, "%s: unknown dtype", who);
    const int32_t function = mode & 0xFF;
    if ((function != EB_SOFTMAX && function != EB_SIGMOID) || (mode & ~(0xFF | EB_RENORMALIZE | EB_GROUP_PAIR)) != 0)
        return fail(EB_ERR_INVALID, "%s: unknown mode", who);
    if (groups < 1 || top_groups < 1 || top_groups > groups || E % groups != 0)
        return fail(EB_ERR_INVALID, "%s: groups must divide E, with 1 <= top_groups <= groups", who);
    if ((mode & EB_GROUP_PAIR) && E / groups < 2) return fail(EB_ERR_INVALID, "%s: pairs need groups of two or more experts", who);
    if (shard_lo < 0 || shard_hi < shard_lo || shard_hi > E) return fail(EB_ERR_INVALID, "%s: bad shard range", who);
    if (!offsets && (tokens || slots)) return fail(EB_ERR_INVALID, "%s: tokens or slots without offsets", who);
    if (E > kMostExperts || K > kMostTop || groups > kMostGroups)
        return fail(EB_ERR_UNSUPPORTED, "%s: more than 1024 experts, 64 per token or 32 groups", who);
    if (N > (int64_t)std::numeric_limits<int32_t>::max() / K) return fail(EB_ERR_UNSUPPORTED, "%s: N * K exceeds 2^31 - 1", who);
    if (N > 1 && ld < E) return fail(EB_ERR_INVALID, "%s: ld below E", who);
    if (N > 0 && (!scores || !ids || !weights)) return fail(EB_ERR_INVALID, "%s: NULL scores, ids or weights", who);
    if (N > 0 && offsets && (!tokens || !slots)) return fail(EB_ERR_INVALID, "%s: NULL tokens or slots", who);
    const int32_t held = shard_hi - shard_lo;
    const size_t needed = offsets ? workspace_of(N, K, held) : 0;
    if (needed > 0 && (!workspace || workspace_bytes < needed || (uintptr_t)workspace % 4))
        return fail(EB_ERR_INVALID, "%s: workspace missing, too small or misaligned", who);

    const hipStream_t s = (hipStream_t)stream;
    if (N == 0) {
        if (!offsets) return EB_OK;
        int32_t n = held + 1;
        void *args[] = {&offsets, &n};
        const hipError_t err = hipLaunchKernel((const void *)eb_route_none, dim3(1), dim3(kThreads), args, 0, s);
        return err == hipSuccess ? EB_OK : fail(EB_ERR_HIP, "%s: kernel launch failed: %s", who, hipGetErrorString(err));
    }
    RouteArgs a{};
    a.scores = scores;
    a.bias = bias;
    a.ld = ld;
    a.N = N;
    a.E = E;
    a.K = K;
    a.sigmoid = function == EB_SIGMOID;
    a.renormalize = (mode & EB_RENORMALIZE) != 0;
    a.pair = (mode & EB_GROUP_PAIR) != 0 && groups > 1;
    a.groups = groups;
    a.top_groups = top_groups;
    a.group_size = E / groups;
    a.group_magic = (1u << 20) / (uint32_t)a.group_size + 1;
    a.scale = scale;
    a.lo = shard_lo;
    a.held = held;
    a.ids = ids;
    a.weights = weights;
    a.offsets = offsets;
    a.tokens = tokens;
    a.slots = slots;
    a.counts = needed > 0 ? (uint32_t *)workspace : nullptr;
    a.chunks = chunks_of(N);
    const bool few = is_few(N, E, K);
    void *kernel = dtype == EB_F32 ? choose_kernel<float>(few, N, E, K) : dtype == EB_F16 ? choose_kernel<_Float16>(few, N, E, K) : choose_kernel<Bf16>(few, N, E, K);
    void *args[] = {&a};
    auto launch = [&](void *f, int64_t grid, int threads) {
        return hipLaunchKernel(f, dim3((unsigned)grid), dim3((unsigned)threads), args, 0, s);
    };
    // Chunks; few pairs, which are not counted by chunk, by what a workgroup takes at once.
    a.each = N * K <= kFewPairs ? kChooseThreads / choose_lanes(E, K) : kTokens;
    const int64_t grid = (N + a.each - 1) / a.each;
    if (grid > std::numeric_limits<uint32_t>::max() / kChooseThreads)
        return fail(EB_ERR_UNSUPPORTED, "%s: more tokens than one launch holds", who);
    hipError_t err = few ? launch(kernel, 1, kAllThreads) : launch(kernel, grid, kChooseThreads);
    if (err == hipSuccess && offsets && !few) {
        if (!a.counts) {
            err = launch((void *)eb_route_place_few, (N * K + kPart - 1) / kPart, kAllThreads);
        } else {
            if (held > 0) err = launch((void *)eb_route_scan, (held + kWaves - 1) / kWaves, kThreads);
            if (err == hipSuccess) err = launch((void *)eb_route_place, a.chunks, kThreads);
        }
    }
    if (err != hipSuccess) return fail(EB_ERR_HIP, "%s: kernel launch failed: %s", who, hipGetErrorString(err));
    return EB_OK;
}

} // namespace

extern "C" {

int eb_route_experts_workspace(int64_t N, int32_t E, int32_t K, int32_t shard_lo, int32_t shard_hi, size_t *bytes)
{
    if (!bytes || N < 0 || K < 1 || K > E || shard_lo < 0 || shard_hi < shard_lo || shard_hi > E)
        return fail(EB_ERR_INVALID, "eb_route_experts_workspace: NULL bytes or a bad size");
    if (E > kMostExperts || K > kMostTop || N > (int64_t)std::numeric_limits<int32_t>::max() / K)
        return fail(EB_ERR_UNSUPPORTED, "eb_route_experts_workspace: more than 1024 experts, 64 per token or 2^31 - 1 pairs");
    *bytes = workspace_of(N, K, shard_hi - shard_lo);
    return EB_OK;
}

int eb_route_experts(int64_t N, int32_t E, int32_t K, const void *scores, int32_t dtype, int64_t ld, const float *bias,
                     int32_t mode, int32_t groups, int32_t top_groups, float scale, int32_t shard_lo, int32_t shard_hi,
                     int32_t *ids, float *weights, int32_t *offsets, int32_t *tokens, int32_t *slots, void *workspace,
                     size_t workspace_bytes, void *stream)
{
    try {
        return route_impl("eb_route_experts", N, E, K, scores, dtype, ld, bias, mode, groups, top_groups, scale, shard_lo,
                          shard_hi, ids, weights, offsets, tokens, slots, workspace, workspace_bytes, stream);
    } catch (...) {
        return eb_detail::unexpected_exception("eb_route_experts");
    }
}

} // extern "C"
