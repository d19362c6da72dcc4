// Which blocks a token attends to: every block's sketch against the token's queries, then the best ones in order.
//
// The scores are products of 8-bit whole numbers on the matrix cores (v_mfma_i32_16x16x64_i8: 16 blocks x 16 tokens; the group's queries are
// summed first and taken apart again into signed digits, lo + 256 hi + 65536 top), so they do not depend on an order of summation; they stay in LDS.  The `top` best are
// those at or above a threshold, which is found from its highest bit on by counting (ballots), and the list comes out in order by ballots, as the
// kept lists of masks are made.
//   k_select: 16 (4) tokens a workgroup; a wave finds one token's threshold.  Prompts.
//   k_select_one: one token a workgroup of 16 waves, the threshold eight bits a round by counting their values in LDS.  Single tokens, where
//     the chain of dependent steps is all that counts, and sequences so long that more tokens' scores do not fit LDS.
#include "fc_attn_internal.hpp"

namespace fc {

namespace {

constexpr int kThreads = 256, kThreadsOne = 1024;

struct SelectArgs {
    KvGeom kv;
    const uint16_t *q;
    int64_t q_row, q_head;
    int32_t group, wide, first, last, top, tiles, stride;   // stride: scores of a token in LDS
    int32_t *selected;
    int32_t *clear;
    int32_t n_clear;
};

// Larger floats have larger keys (no NaN).
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t u = __float_as_uint(v + 0.f);            // (-0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int DT> __device__ __forceinline__ float element(const uint4 &x, int j)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    return bits_to_float<DT>((uint16_t)(w[j >> 1] >> (16 * (j & 1))));
}
// The digits of a sum of rounded queries.  A rounded query is at most 255 (127 below the units' bound), so two digits hold the sums of groups of up to kTwoDigits
// heads (255 * 127 = 32385 of 32639) and three those of up to kMostGroup; two digits' products with sketches of 256 channels add up in 32 bits, three in 64.
constexpr int kTwoDigits = 127;
__device__ __forceinline__ int digit_of(int sum, int nth)
{
    const int lo = (int8_t)sum, hi = (int8_t)((sum - lo) >> 8);
    return nth == 0 ? lo : nth == 1 ? hi : (sum - lo - 256 * hi) >> 16;
}

__device__ __forceinline__ bool finite(float v) { return __builtin_fabsf(v) < __builtin_inff(); }

template <int DT> __device__ __forceinline__ float largest(const uint4 &x, float most)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float v = element<DT>(x, j);
        most = finite(v) ? fmaxf(most, __builtin_fabsf(v)) : most;
    }
    return most;
}

// The sketches of 16 blocks: a lane's share, and (lanes alike in lane % 16) a block's weight.
template <int DP> struct Sketches {
    static constexpr int kChunks = kSketch<DP> / 64;
    i32x4_t x[kChunks];
    float weight;
    __device__ __forceinline__ void bring(const KvGeom &g, int b, int h, int first, int end)
    {
        const int lane = threadIdx.x & 63, block = first + (lane & 15);
        const int32_t pool = pool_block(g, b, min(block, end - 1));
        const int64_t unit = unit_of(g, max(pool, 0), h);
        // (of a block that is not there another one's sketch, without weight)
        weight = g.weights[unit];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) x[c] = *reinterpret_cast<const i32x4_t *>(g.sketches + unit * kSketch<DP> + 64 * c + (lane >> 4) * 16);
        if (pool < 0) weight = 0.f;
    }
    // keys of blocks 4 (lane / 16) + i and token lane % 16
    template <int DIGITS> __device__ __forceinline__ void score(const i32x4_t (&q)[DIGITS][kChunks], uint32_t (&keys)[4]) const
    {
        i32x4_t sum[DIGITS];
#pragma unroll
        for (int n = 0; n < DIGITS; ++n) {
            sum[n] = i32x4_t{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < kChunks; ++c) sum[n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[c], q[n][c], sum[n], 0, 0, 0);
        }
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float total;
            if constexpr (DIGITS == 2) total = (float)(256 * sum[1][i] + sum[0][i]);
            else total = (float)(65536 * (int64_t)sum[2][i] + 256 * (int64_t)sum[1][i] + sum[0][i]);
            keys[i] = key_of(total * __shfl(weight, (lane >> 4) * 4 + i));
        }
    }
};

// The first entries, the last ones, and whole lists of tokens with few blocks.  Returns whether blocks have to be chosen.
__device__ __forceinline__ bool fixed_entries(const SelectArgs &a, int own, int32_t *out, int at, int step)
{
    const int width = a.first + a.last + a.top;
    if (own + 1 <= width) {
        for (int i = at; i < width; i += step) out[i] = i <= own ? i : -1;
        return false;
    }
    for (int i = at; i < a.first; i += step) out[i] = i;
    for (int i = at; i < a.last; i += step) out[a.first + a.top + i] = own - a.last + 1 + i;
    return a.top != 0;
}

// Entries of candidates from .. to - 1: those above the threshold, and those at it while `ties` of them are not yet used up.
__device__ __forceinline__ void write_entries(const uint32_t *keys, int from, int to, uint32_t threshold, int ties, int32_t first, int32_t *out)
{
    const int lane = threadIdx.x & 63;
    const uint64_t below = (1ull << lane) - 1;
    for (int i = from; i < to; i += 64) {
        const bool inside = i + lane < to;
        const uint32_t key = inside ? keys[i + lane] : 0;
        const uint64_t equals = __ballot(inside && key == threshold);
        const bool take = inside && (key > threshold || (key == threshold && (int)__popcll(equals & below) < ties));
        const uint64_t takes = __ballot(take);
        if (take) out[__popcll(takes & below)] = first + i + lane;
        ties -= (int)__popcll(equals);
        out += __popcll(takes);
    }
}

// A threshold that `top` of the lanes' keys or more are at or above (exactly as many, or the largest), bit by bit.
__device__ __forceinline__ uint32_t threshold_of_lanes(uint32_t key, int top)
{
    uint32_t threshold = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t trial = threshold | 1u << bit;
        const int c = (int)__popcll(__ballot(key >= trial));
        if (c >= top) threshold = trial;
        if (c == top) break;
    }
    return threshold;
}

// The same for n keys in LDS, by one wave; above: keys above it.  `few`: 64 words of the wave's own.
// Up to 64: the lanes' largest keys give a threshold that is no higher than the one looked for, and few keys are at or above that one, which then are one a
// lane: two searches of one key a lane in place of one of all.
template <int REGS> __device__ __forceinline__ uint32_t threshold_of(const uint32_t *keys, int n, int top, uint32_t *few, int &above)
{
    const int lane = threadIdx.x & 63;
    uint32_t held[REGS > 0 ? REGS : 1];
#pragma unroll
    for (int r = 0; r < REGS; ++r) held[r] = 64 * r + lane < n ? keys[64 * r + lane] : 0;      // (no key is 0: no score is that low)
    auto each = [&](auto f) {
        if constexpr (REGS > 0) {
#pragma unroll
            for (int r = 0; r < REGS; ++r) f(held[r]);
        } else {
            for (int i = 0; i < n; i += 64) f(i + lane < n ? keys[i + lane] : 0);
        }
    };
    auto count = [&](uint32_t trial) {
        int c = 0;
        each([&](uint32_t key) { c += (int)__popcll(__ballot(key >= trial)); });
        return c;
    };
    // (the largest key there is: a NaN, as the weight of a block that was never written may be)
    auto count_above = [&](uint32_t threshold) { return threshold == ~0u ? 0 : count(threshold + 1); };
    uint32_t threshold = 0;
    if (top <= 64) {
        uint32_t largest_key = 0;
        each([&](uint32_t key) { largest_key = max(largest_key, key); });
        const uint32_t least = max(threshold_of_lanes(largest_key, top), 1u);
        const int some = count(least);
        if (some == top) {
            above = count_above(least);
            return least;
        }
        if (some <= 64) {
            const uint64_t below = (1ull << lane) - 1;
            int at = 0;
            each([&](uint32_t key) {
                const uint64_t takes = __ballot(key >= least);
                if (key >= least) few[at + __popcll(takes & below)] = key;
                at += (int)__popcll(takes);
            });
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const uint32_t key = lane < some ? few[lane] : 0;
            threshold = threshold_of_lanes(key, top);
            above = (int)__popcll(__ballot(key > threshold));
            return threshold;
        }
    }
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t trial = threshold | 1u << bit;
        const int c = count(trial);
        if (c >= top) threshold = trial;
        if (c == top) break;
    }
    above = count_above(threshold);
    return threshold;
}

// Bound by the counting of the thresholds (a compare and a ballot for 64 scores a bit, at most 32 bits, scalar additions beside them).  4096 tokens, 8 heads of 128 with 4 queries
// each, up to 512 blocks: 63 us.
template <int DT, int DP, int QT, int DIGITS> __global__ __launch_bounds__(kThreads) void k_select(SelectArgs a)
{
    constexpr int SP = kSketch<DP>, kChunks = SP / 64, kShare = kThreads / QT;        // threads of a token
    extern __shared__ uint32_t lds_keys[];
    __shared__ __align__(16) int8_t q8[DIGITS][QT][SP];             // lo, hi and top
    __shared__ uint32_t amax[QT], few[kThreads / 64][64];
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < a.n_clear; i += gridDim.x * kThreads) a.clear[i] = 0;
    const KvGeom &g = a.kv;
    uint32_t at = blockIdx.x;
    const int tile = at % a.tiles;
    at /= a.tiles;
    const int h = at % g.kv_heads, b = at / g.kv_heads;
    const Sequence s = sequence_of(g, b);
    const int token0 = tile * QT, tokens = min(s.n - token0, QT);
    if (tokens <= 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
    const int last_pos = s.pos0 + token0 + tokens - 1, width = a.first + a.last + a.top;
    // blocks that a score is wanted for: below `scored`; none where every token takes all its blocks
    const int own_most = last_pos < 0 ? -1 : last_pos / kBlock;
    const int scored = own_most + 1 <= width || a.top == 0 ? 0 : own_most - a.last + 1;

    if (scored > 0) {
        const int mine = threadIdx.x / kShare, share = threadIdx.x % kShare;
        if (threadIdx.x < QT) amax[threadIdx.x] = 0;
        __syncthreads();
        const uint16_t *const q = a.q + (int64_t)(s.row0 + token0 + mine) * a.q_row + (int64_t)h * a.group * a.q_head;
        if (mine < tokens) {
            float most = 0.f;
            for (int i = share; i < a.group * (DP / 8); i += kShare)
                most = largest<DT>(load8(q + (int64_t)(i / (DP / 8)) * a.q_head, i % (DP / 8) * 8, g.d, a.wide), most);
            atomicMax(&amax[mine], __float_as_uint(most));
        }
        __syncthreads();
        const float inverse = pow2_of(-unit_exponent(__uint_as_float(amax[mine])));
        for (int c = share; c < SP / 8; c += kShare) {       // (behind head_dim: zeros)
            int sum[8] = {};
            if (mine < tokens)
                for (int head = 0; head < a.group; ++head) {
                    const uint4 x = load8(q + head * a.q_head, 8 * c, g.d, a.wide);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float v = element<DT>(x, j);
                        sum[j] += finite(v) ? (int)__builtin_rintf(v * inverse) : 0;
                    }
                }
#pragma unroll
            for (int n = 0; n < DIGITS; ++n)
#pragma unroll
                for (int j = 0; j < 8; ++j) q8[n][mine][8 * c + j] = (int8_t)digit_of(sum[j], n);
        }
        __syncthreads();
        i32x4_t digits[DIGITS][kChunks];
#pragma unroll
        for (int n = 0; n < DIGITS; ++n)
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                digits[n][c] = i32x4_t{0, 0, 0, 0};
                if (col < QT) digits[n][c] = *reinterpret_cast<const i32x4_t *>(&q8[n][col % QT][64 * c + 16 * quarter]);
            }
        auto put = [&](const Sketches<DP> &x, int first) {
            uint32_t keys[4];
            x.score(digits, keys);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col < QT && first + quarter * 4 + i < scored) lds_keys[col * a.stride + first + quarter * 4 + i] = keys[i];
        };
        for (int first = wave * 16; first < scored; first += 128) {
            Sketches<DP> x0, x1;
            x0.bring(g, b, h, first, scored);
            x1.bring(g, b, h, first + 64, scored);
            put(x0, first);
            put(x1, first + 64);
        }
        __syncthreads();
    }

    for (int mine = wave; mine < tokens; mine += kThreads / 64) {
        const int pos = s.pos0 + token0 + mine, own = pos < 0 ? -1 : pos / kBlock;
        int32_t *const out = a.selected + ((int64_t)(s.row0 + token0 + mine) * g.kv_heads + h) * width;
        if (!fixed_entries(a, own, out, lane, 64)) continue;
        const int candidates = own + 1 - a.first - a.last;      // (more than top)
        const uint32_t *const keys = lds_keys + mine * a.stride + a.first;
        int above;
        const uint32_t threshold = candidates <= 256 ? threshold_of<4>(keys, candidates, a.top, few[wave], above) :
                                   candidates <= 512 ? threshold_of<8>(keys, candidates, a.top, few[wave], above) :
                                   candidates <= 1024 ? threshold_of<16>(keys, candidates, a.top, few[wave], above) : threshold_of<0>(keys, candidates, a.top, few[wave], above);
        write_entries(keys, 0, candidates, threshold, a.top - above, a.first, out + a.first);
    }
}

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int sum_up_to(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);     // row_shr by 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);     // the last lane of a row to the next row
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);     // ... of the first half to the second
    return v;
}

// One token over 512 blocks, 8 heads of 128: 8.5 us; 16 tokens over up to 1016 blocks: 13.4 us (queries, sketches, two to four rounds of counting, the list: dependent steps).
template <int DT, int DP> __global__ __launch_bounds__(kThreadsOne) void k_select_one(SelectArgs a)
{
    constexpr int SP = kSketch<DP>, kChunks = SP / 64, kWaves = kThreadsOne / 64;
    extern __shared__ uint32_t lds_keys[];
    __shared__ __align__(16) int bins[4][256];
    __shared__ __align__(16) int8_t q8[3][SP];      // lo, hi, top
    __shared__ int sums[SP], aboves[kWaves], equals[kWaves];
    __shared__ uint32_t amax;
    for (int i = blockIdx.x * kThreadsOne + threadIdx.x; i < a.n_clear; i += gridDim.x * kThreadsOne) a.clear[i] = 0;
    const KvGeom &g = a.kv;
    uint32_t at = blockIdx.x;
    const int token = at % a.tiles;
    at /= a.tiles;
    const int h = at % g.kv_heads, b = at / g.kv_heads;
    const Sequence s = sequence_of(g, b);
    if (token >= s.n) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;
    const int pos = s.pos0 + token, own = pos < 0 ? -1 : pos / kBlock, width = a.first + a.last + a.top;
    int32_t *const out = a.selected + ((int64_t)(s.row0 + token) * g.kv_heads + h) * width;
    if (!fixed_entries(a, own, out, threadIdx.x, kThreadsOne)) return;
    const int scored = own - a.last + 1, candidates = scored - a.first;
    bins[threadIdx.x >> 8][threadIdx.x & 255] = 0;

    for (int i = threadIdx.x; i < SP; i += kThreadsOne) sums[i] = 0;
    if (threadIdx.x == 0) amax = 0;

    Sketches<DP> x;
    x.bring(g, b, h, 16 * wave, scored);
    // The queries, an element a thread (of more than 1024 the others are read twice)
    const uint16_t *const q = a.q + (int64_t)(s.row0 + token) * a.q_row + (int64_t)h * a.group * a.q_head;
    const int elements = a.group * DP;
    auto query = [&](int i) {
        const int head = i / DP, c = i % DP;
        const float v = i < elements && c < g.d ? bits_to_float<DT>(q[head * a.q_head + c]) : 0.f;
        return finite(v) ? v : 0.f;
    };
    const float mine = query(threadIdx.x);
    float most = __builtin_fabsf(mine);
    for (int i = threadIdx.x + kThreadsOne; i < elements; i += kThreadsOne) most = fmaxf(most, __builtin_fabsf(query(i)));
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    most = max_over_16(max_over_32(most));
    __syncthreads();
    if (lane == 0 && most > 0.f) atomicMax(&amax, __float_as_uint(most));
    __syncthreads();
    const float inverse = pow2_of(-unit_exponent(__uint_as_float(amax)));
    for (int i = threadIdx.x; i < elements; i += kThreadsOne)
        atomicAdd(&sums[i % DP], (int)__builtin_rintf((i < kThreadsOne ? mine : query(i)) * inverse));
    __syncthreads();
    if (threadIdx.x < SP) {
        const int sum = sums[threadIdx.x];
#pragma unroll
        for (int n = 0; n < 3; ++n) q8[n][threadIdx.x] = (int8_t)digit_of(sum, n);
    }
    __syncthreads();
    i32x4_t parts[kChunks];         // columns 0 to 2 of the product's operand are lo, hi and top
    const bool three = a.group > kTwoDigits;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        parts[c] = i32x4_t{0, 0, 0, 0};
        if (col < 3) parts[c] = *reinterpret_cast<const i32x4_t *>(&q8[col][64 * c + 16 * quarter]);
    }
    for (int first = 16 * wave; first < scored; first += 16 * kWaves) {
        i32x4_t sum = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < kChunks; ++c) sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(x.x[c], parts[c], sum, 0, 0, 0);
        const float weight = x.weight;
        if (first + 16 * kWaves < scored) x.bring(g, b, h, first + 16 * kWaves, scored);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int hi = __builtin_amdgcn_update_dpp(0, sum[i], 0x101, 0xf, 0xf, false);      // row_shl by 1: column 1's
            const int top = __builtin_amdgcn_update_dpp(0, sum[i], 0x102, 0xf, 0xf, false);     // by 2
            const int to = first + quarter * 4 + i;
            const float w = __shfl(weight, quarter * 4 + i);
            const float total = three ? (float)(65536 * (int64_t)top + 256 * (int64_t)hi + sum[i]) : (float)(256 * hi + sum[i]);
            if (col == 0 && to < scored) lds_keys[to] = key_of(total * w);
        }
    }
    __syncthreads();

    // The threshold, eight bits a round: how many keys have each value of them, and the value at which the `top` best are together.  Every wave finds it.
    // A wave looks after its part of the candidates.
    const uint32_t *const keys = lds_keys + a.first;
    const int part = (candidates + 64 * kWaves - 1) / (64 * kWaves) * 64, from = min(wave * part, candidates), to = min(from + part, candidates);
    uint32_t threshold = 0;
    int wanted = a.top;             // of the keys that agree with the threshold so far
#pragma unroll
    for (int round = 0; round < 4; ++round) {
        const int shift = 24 - 8 * round;
        for (int i = from + lane; i < to; i += 64) {
            const uint32_t key = keys[i];
            if (round == 0 || (key ^ threshold) >> (shift + 8) == 0) atomicAdd(&bins[round][key >> shift & 255], 1);
        }
        __syncthreads();
        const int4 four = *reinterpret_cast<const int4 *>(&bins[round][252 - 4 * lane]);      // lane 0 has the largest values
        const int mine_sum = four.x + four.y + four.z + four.w, up_to = sum_up_to(mine_sum);
        const int at_lane = __ffsll((unsigned long long)__ballot(up_to >= wanted)) - 1;
        int before = __builtin_amdgcn_readlane(up_to - mine_sum, at_lane);
        const int n[4] = {__builtin_amdgcn_readlane(four.w, at_lane), __builtin_amdgcn_readlane(four.z, at_lane), __builtin_amdgcn_readlane(four.y, at_lane),
                          __builtin_amdgcn_readlane(four.x, at_lane)};
        int value = 255 - 4 * at_lane, here = n[0];
#pragma unroll
        for (int j = 1; j < 4; ++j)
            if (before + here < wanted) {
                before += here;
                here = n[j];
                --value;
            }
        threshold |= (uint32_t)value << shift;
        wanted -= before;
        if (here == wanted) break;  // all of these
    }

    int above = 0, same = 0;
    for (int i = from; i < to; i += 64) {
        const uint32_t key = i + lane < to ? keys[i + lane] : 0;
        above += (int)__popcll(__ballot(key > threshold));
        same += (int)__popcll(__ballot(i + lane < to && key == threshold));
    }
    if (lane == 0) {
        aboves[wave] = above;
        equals[wave] = same;
    }
    __syncthreads();
    int above_before = 0, same_before = 0, above_all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        above_all += aboves[w];
        above_before += w < wave ? aboves[w] : 0;
        same_before += w < wave ? equals[w] : 0;
    }
    const int ties = a.top - above_all;         // of those at the threshold, the lowest numbers
    write_entries(keys, from, to, threshold, ties - same_before, a.first, out + a.first + above_before + min(same_before, ties));
}

template <int DT, int DP, int QT, int DIGITS> hipError_t run_tokens(SelectArgs a, hipStream_t s)
{
    a.tiles = (a.kv.max_new + QT - 1) / QT;
    const size_t lds = (size_t)QT * a.stride * sizeof(uint32_t);
    const dim3 grid((uint32_t)((int64_t)a.kv.batch * a.kv.kv_heads * a.tiles));
    if (lds > 32 * 1024) {
        hipError_t e;
        if constexpr (QT == 1) e = raise_lds<k_select_one<DT, DP>>((size_t)128 * 1024);
        else e = raise_lds<k_select<DT, DP, QT, DIGITS>>((size_t)128 * 1024);
        if (e != hipSuccess) return e;
    }
    if constexpr (QT == 1) k_select_one<DT, DP><<<grid, kThreadsOne, lds, s>>>(a);
    else k_select<DT, DP, QT, DIGITS><<<grid, kThreads, lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, int DP> hipError_t run_dim(const SelectArgs &a, hipStream_t s)
{
    const int tokens = select_tokens(a.kv);
    if (tokens == 1) return run_tokens<DT, DP, 1, 3>(a, s);
    // (apart because the third digit's registers cost two of eight waves a SIMD)
    if (a.group > kTwoDigits) return tokens == 4 ? run_tokens<DT, DP, 4, 3>(a, s) : run_tokens<DT, DP, 16, 3>(a, s);
    return tokens == 4 ? run_tokens<DT, DP, 4, 2>(a, s) : run_tokens<DT, DP, 16, 2>(a, s);
}

template <int DT> hipError_t run_type(const SelectArgs &a, hipStream_t s)
{
    switch (a.kv.dp) {
    case 64: return run_dim<DT, 64>(a, s);
    case 96: return run_dim<DT, 96>(a, s);
    case 128: return run_dim<DT, 128>(a, s);
    case 192: return run_dim<DT, 192>(a, s);
    default: return run_dim<DT, 256>(a, s);
    }
}

} // namespace

hipError_t launch_select(const KvGeom &g, int dtype, const uint16_t *q, int64_t q_row, int64_t q_head, int heads, bool wide, int first, int last,
                         int top, int32_t *selected, int32_t *clear, int32_t n_clear, hipStream_t s)
{
    const int stride = select_stride(g);
    const SelectArgs a = {g, q, q_row, q_head, heads / g.kv_heads, wide, first, last, top, 0, stride, selected, clear, n_clear};
    return dtype == FC_BF16 ? run_type<FC_BF16>(a, s) : run_type<FC_F16>(a, s);
}

} // namespace fc
