// Which blocks a token attends to: every block's sketch against the token's queries, then the best ones in order.
//
// A workgroup takes up to 16 tokens of one sequence and one key head.  The scores are products of 8-bit whole numbers on the matrix
// cores (v_mfma_i32_16x16x64_i8: 16 blocks x 16 tokens; the group's queries are summed first and taken apart again into 128 hi + lo),
// so they do not depend on an order of summation; they stay in LDS.  A wave then picks one token's blocks: the threshold bit by
// bit, and the list in order by ballots, as the kept lists of masks are made.
#include "fc_attn_internal.hpp"

namespace fc {

namespace {

constexpr int kThreads = 256;

struct SelectArgs {
    KvGeom kv;
    const uint16_t *q;
    int64_t q_row, q_head;
    int32_t group, wide, first, last, top, tiles, stride;   // stride: scores of a token in LDS
    int32_t *selected;
};

// Larger floats have larger keys (no NaN).
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t u = __float_as_uint(v + 0.f);            // (-0 is 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int DT, int DP, int QT> __global__ __launch_bounds__(kThreads) void k_select(SelectArgs a)
{
    constexpr int kChunks = DP / 64, kShare = kThreads / QT;        // threads of a token
    extern __shared__ uint32_t lds_keys[];
    __shared__ __align__(16) int8_t q8[2][QT][DP];                  // hi, lo
    __shared__ uint32_t amax[QT];
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
    // blocks that a score is wanted for: first .. scored - 1, unless every token takes all its blocks
    const int own_most = last_pos < 0 ? -1 : last_pos / kBlock;
    const int scored = own_most + 1 <= width || a.top == 0 ? 0 : own_most - a.last + 1;

    if (scored > a.first) {
        const int mine = threadIdx.x / kShare, share = threadIdx.x % kShare;
        if (threadIdx.x < QT) amax[threadIdx.x] = 0;
        __syncthreads();
        const uint16_t *const q = a.q + (int64_t)(s.row0 + token0 + mine) * a.q_row + (int64_t)h * a.group * a.q_head;
        if (mine < tokens) {
            float most = 0.f;
            for (int i = share; i < a.group * (DP / 8); i += kShare) {
                const uint4 x = load8(q + (int64_t)(i / (DP / 8)) * a.q_head, i % (DP / 8) * 8, g.d, a.wide);
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float v = __builtin_fabsf(bits_to_float<DT>((uint16_t)(w[j >> 1] >> (16 * (j & 1)))));
                    most = v < __builtin_inff() ? fmaxf(most, v) : most;
                }
            }
            atomicMax(&amax[mine], __float_as_uint(most));
        }
        __syncthreads();
        const float inverse = pow2_of(-unit_exponent(__uint_as_float(amax[mine])));
        for (int c = share; c < DP / 8; c += kShare) {
            int sum[8] = {};
            if (mine < tokens)
                for (int head = 0; head < a.group; ++head) {
                    const uint4 x = load8(q + head * a.q_head, 8 * c, g.d, a.wide);
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float v = bits_to_float<DT>((uint16_t)(w[j >> 1] >> (16 * (j & 1))));
                        sum[j] += __builtin_fabsf(v) < __builtin_inff() ? (int)__builtin_rintf(v * inverse) : 0;
                    }
                }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                q8[0][mine][8 * c + j] = (int8_t)(sum[j] >> 7);
                q8[1][mine][8 * c + j] = (int8_t)(sum[j] & 127);
            }
        }
        __syncthreads();
        i32x4_t hi[kChunks], lo[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            hi[c] = lo[c] = i32x4_t{0, 0, 0, 0};
            if (col < QT) {
                hi[c] = *reinterpret_cast<const i32x4_t *>(&q8[0][col % QT][64 * c + 16 * quarter]);
                lo[c] = *reinterpret_cast<const i32x4_t *>(&q8[1][col % QT][64 * c + 16 * quarter]);
            }
        }
        for (int first = wave * 16; first < scored; first += 64) {
            const int block = first + col;
            const int32_t pool = block < scored ? pool_block(g, b, block) : -1;
            const int64_t unit = unit_of(g, max(pool, 0), h);
            const float weight = pool < 0 ? 0.f : g.weights[unit];
            i32x4_t up = {0, 0, 0, 0}, down = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                i32x4_t x = {0, 0, 0, 0};
                if (pool >= 0) x = *reinterpret_cast<const i32x4_t *>(g.sketches + unit * DP + 64 * c + 16 * quarter);
                up = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, hi[c], up, 0, 0, 0);
                down = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, lo[c], down, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w = __shfl(weight, quarter * 4 + i);
                const int to = first + quarter * 4 + i;
                if (col < QT && to < scored) lds_keys[col * a.stride + to] = key_of((float)(128 * up[i] + down[i]) * w);
            }
        }
        __syncthreads();
    }

    for (int mine = wave; mine < tokens; mine += kThreads / 64) {
        const int pos = s.pos0 + token0 + mine, own = pos < 0 ? -1 : pos / kBlock;
        int32_t *const out = a.selected + ((int64_t)(s.row0 + token0 + mine) * g.kv_heads + h) * width;
        if (own + 1 <= width) {
            for (int i = lane; i < width; i += 64) out[i] = i <= own ? i : -1;
            continue;
        }
        for (int i = lane; i < a.first; i += 64) out[i] = i;
        for (int i = lane; i < a.last; i += 64) out[a.first + a.top + i] = own - a.last + 1 + i;
        if (a.top == 0) continue;
        const int candidates = own + 1 - a.first - a.last;      // (more than top)
        const uint32_t *const keys = lds_keys + mine * a.stride + a.first;
        uint32_t threshold = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t trial = threshold | 1u << bit;
            int count = 0;
            for (int i = 0; i < candidates; i += 64) count += __popcll(__ballot(i + lane < candidates && keys[i + lane] >= trial));
            if (count >= a.top) threshold = trial;
        }
        int above = 0;
        for (int i = 0; i < candidates; i += 64) above += __popcll(__ballot(i + lane < candidates && keys[i + lane] > threshold));
        const int ties = a.top - above;                          // of those at the threshold, the lowest numbers
        int seen = 0, put = a.first;
        const uint64_t below = (1ull << lane) - 1;
        for (int i = 0; i < candidates; i += 64) {
            const uint32_t key = i + lane < candidates ? keys[i + lane] : 0;
            const bool equal = i + lane < candidates && key == threshold;
            const uint64_t equals = __ballot(equal);
            const bool take = (i + lane < candidates && key > threshold) || (equal && seen + __popcll(equals & below) < ties);
            const uint64_t takes = __ballot(take);
            if (take) out[put + __popcll(takes & below)] = a.first + i + lane;
            seen += __popcll(equals);
            put += __popcll(takes);
        }
    }
}

template <int DT, int DP, int QT> hipError_t run_tokens(SelectArgs a, hipStream_t s)
{
    a.tiles = (a.kv.max_new + QT - 1) / QT;
    const size_t lds = (size_t)QT * a.stride * sizeof(uint32_t);
    if (lds > 32 * 1024) {
        const hipError_t e = raise_lds<k_select<DT, DP, QT>>((size_t)128 * 1024);
        if (e != hipSuccess) return e;
    }
    k_select<DT, DP, QT><<<dim3((uint32_t)((int64_t)a.kv.batch * a.kv.kv_heads * a.tiles)), kThreads, lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, int DP> hipError_t run_dim(const SelectArgs &a, hipStream_t s)
{
    // as many tokens a workgroup as their scores have room in LDS; single tokens alone
    if (a.kv.max_new == 1 || a.stride > 8192) return run_tokens<DT, DP, 1>(a, s);
    return a.stride > 2048 ? run_tokens<DT, DP, 4>(a, s) : run_tokens<DT, DP, 16>(a, s);
}

template <int DT> hipError_t run_type(const SelectArgs &a, hipStream_t s)
{
    switch (a.kv.dp) {
    case 64: return run_dim<DT, 64>(a, s);
    case 128: return run_dim<DT, 128>(a, s);
    case 192: return run_dim<DT, 192>(a, s);
    default: return run_dim<DT, 256>(a, s);
    }
}

} // namespace

hipError_t launch_select(const KvGeom &g, int dtype, const uint16_t *q, int64_t q_row, int64_t q_head, int heads, bool wide, int first, int last,
                         int top, int32_t *selected, hipStream_t s)
{
    const int stride = (int)align_up((size_t)(g.max_len + kBlock - 1) / kBlock, 16);
    const SelectArgs a = {g, q, q_row, q_head, heads / g.kv_heads, wide, first, last, top, 0, stride, selected};
    return dtype == FC_BF16 ? run_type<FC_BF16>(a, s) : run_type<FC_F16>(a, s);
}

} // namespace fc
