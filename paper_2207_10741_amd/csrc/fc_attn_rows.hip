// Attention of few rows over a long axis: single tokens, and single tokens' lists of blocks.
//
// A workgroup holds 16 or 32 rows (new tokens x the heads of one key head's group) and a piece of the sequence's blocks; its four waves
// take every fourth block each, with a softmax of their own (running maximum and sum), and are joined through LDS.  Pieces are joined by
// k_attend_join.  A block goes from memory to registers in the order the matrix instructions want it (fc_attn_internal.hpp): no LDS and
// no lane exchange on the way, but for the rows' maximum.
#include "fc_attn_internal.hpp"

namespace fc {

namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

// max over the four lanes that hold one row
__device__ __forceinline__ float row_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float row_sum(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

template <int DT, int DP, int MT, bool LIST> __global__ __launch_bounds__(kThreads) void k_attend_rows(AttnArgs a)
{
    constexpr int kChunks = DP / 64, kTiles = DP / 16, kRows = 16 * MT, kPitch = DP + 4;
    extern __shared__ float lds[];
    float *const lds_m = lds, *const lds_l = lds + kWaves * kRows, *const lds_o = lds + 2 * kWaves * kRows;
    const KvGeom &g = a.kv;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;

    uint32_t at = blockIdx.x;
    const int split = at % a.splits;
    at /= a.splits;
    const int tile = at % a.tiles;
    at /= a.tiles;
    const int h = at % g.kv_heads, b = at / g.kv_heads;
    const Sequence s = sequence_of(g, b);

    // row r of the tile: new token i, head `head` of the group
    int token0, head0, rows;
    if constexpr (LIST) {
        const int per_token = (a.group + kRows - 1) / kRows;
        token0 = tile / per_token;
        head0 = tile % per_token * kRows;
        rows = token0 < s.n ? min(a.group - head0, kRows) : 0;
    } else {
        token0 = (int)fast_div((uint32_t)(tile * kRows), a.div_group);
        head0 = tile * kRows - token0 * a.group;
        rows = min(max(s.n * a.group - tile * kRows, 0), kRows);
    }
    if (rows <= 0) return;
    int token[MT], head[MT], last[MT];      // last: the last position that the row attends to
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = 16 * mt + col;
        const int q = (int)fast_div((uint32_t)(head0 + r), a.div_group);
        token[mt] = LIST ? token0 : token0 + q;
        head[mt] = LIST ? head0 + r : head0 + r - q * a.group;
        last[mt] = r < rows ? (a.causal ? s.pos0 + token[mt] : s.len - 1) : -1;
    }
    const int token_last = LIST ? token0 : token0 + (int)fast_div((uint32_t)(head0 + rows - 1), a.div_group);
    const int last_least = a.causal ? s.pos0 + token0 : s.len - 1, last_most = a.causal ? s.pos0 + token_last : s.len - 1;
    int blocks = last_most < 0 ? 0 : last_most / kBlock + 1;
    const int32_t *list = nullptr;
    if constexpr (LIST) {
        list = a.selected + ((int64_t)(s.row0 + token0) * g.kv_heads + h) * a.selected_width;
        blocks = min(blocks, a.selected_width);     // (the selection's count)
    }
    const int active = max((blocks + a.per_split - 1) / a.per_split, 1);
    if (split >= active) return;
    const int end = min(blocks, (split + 1) * a.per_split);

    uint4 q[MT][2 * kChunks];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int c = 0; c < 2 * kChunks; ++c) {
            q[mt][c] = make_uint4(0, 0, 0, 0);
            if (16 * mt + col < rows)
                q[mt][c] = flip_signs(load8(a.q + (s.row0 + token[mt]) * a.q_row + (int64_t)(h * a.group + head[mt]) * a.q_head,
                                            (c >> 1) * 64 + quarter * 16 + (c & 1) * 8, g.d, a.wide), a.signs);
        }

    f32x4_t o[MT][kTiles];
    float m[MT], l[MT], unit_v = 1.f;       // o is in units of the last block's scale
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        m[mt] = -__builtin_inff();
        l[mt] = 0.f;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) o[mt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    for (int j = split * a.per_split + wave; j < end; j += kWaves) {
        const int block = LIST ? list[j] : j;
        const int32_t pool = pool_block(g, b, block);
        if (pool < 0) continue;
        const int64_t unit = unit_of(g, pool, h);
        const uint8_t *const kc = g.codes + unit * (2 * kBlock * DP), *const vc = kc + kBlock * DP;
        const float2 scales = g.scales[unit];
        uint4 kx[4][kChunks], vx[kTiles];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < kChunks; ++c) kx[t][c] = *reinterpret_cast<const uint4 *>(kc + (16 * t + col) * DP + 64 * c + 16 * quarter);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) vx[t] = *reinterpret_cast<const uint4 *>(vc + (16 * t + col) * 64 + 16 * quarter);

        f32x4_t z[MT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) z[mt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const uint4 k0 = codes_to_16<DT>(kx[t][c].x, kx[t][c].y), k1 = codes_to_16<DT>(kx[t][c].z, kx[t][c].w);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    z[mt][t] = mfma16<DT>(k0, q[mt][2 * c], z[mt][t]);
                    z[mt][t] = mfma16<DT>(k1, q[mt][2 * c + 1], z[mt][t]);
                }
            }
        }

        const float to_log2 = a.scale_log2 * scales.x, unit_new = __builtin_fabsf(scales.y);
        const bool partly = block * kBlock + kBlock - 1 > last_least;
        uint4 p[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float most = -__builtin_inff();
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = z[mt][t][i] * to_log2;
                    if (partly) v = block * kBlock + 16 * t + 4 * quarter + i <= last[mt] ? v : -__builtin_inff();
                    z[mt][t][i] = v;
                    most = fmaxf(most, v);
                }
            const float m_new = fmaxf(m[mt], row_max(most));
            const float base = m_new == -__builtin_inff() ? 0.f : m_new;
            const float old = __builtin_amdgcn_exp2f(m[mt] - base);
            m[mt] = m_new;
            float sum = 0.f;
            uint32_t w[8];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    e[i] = __builtin_amdgcn_exp2f(z[mt][t][i] - base);
                    sum += e[i];
                }
                w[2 * t] = pack2<FC_F16>(e[0], e[1]);
                w[2 * t + 1] = pack2<FC_F16>(e[2], e[3]);
            }
            p[mt][0] = make_uint4(w[0], w[1], w[2], w[3]);
            p[mt][1] = make_uint4(w[4], w[5], w[6], w[7]);
            l[mt] = l[mt] * old + sum;
            const float factor = old * fminf(unit_v / unit_new, 0x1p127f);      // (finite: zero stays zero)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) o[mt][t] *= factor;
        }
        unit_v = unit_new;

        if (partly && scales.y < 0.f) {
            // NaN among the values of a block that some rows see in part: a weight of zero does not silence it in a matrix product.  The
            // product runs on zeros in NaN's place, and a second one counts the NaN that a row does see.
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                uint32_t w[8];
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int first = block * kBlock + 16 * t + 4 * quarter + 2 * i;
                        w[2 * t + i] = (first <= last[mt] ? 0x3c00u : 0u) | (first + 1 <= last[mt] ? 0x3c000000u : 0u);
                    }
                const uint4 seen[2] = {make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7])};
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    uint4 clean[2], marks[2];
                    split_nan(codes_to_16<FC_F16>(vx[t].x, vx[t].y), clean[0], marks[0]);
                    split_nan(codes_to_16<FC_F16>(vx[t].z, vx[t].w), clean[1], marks[1]);
                    o[mt][t] = mfma16<FC_F16>(clean[0], p[mt][0], o[mt][t]);
                    o[mt][t] = mfma16<FC_F16>(clean[1], p[mt][1], o[mt][t]);
                    f32x4_t count = {0.f, 0.f, 0.f, 0.f};
                    count = mfma16<FC_F16>(marks[0], seen[0], count);
                    count = mfma16<FC_F16>(marks[1], seen[1], count);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[mt][t][i] = count[i] > 0.f ? __builtin_nanf("") : o[mt][t][i];
                }
            }
            continue;
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const uint4 v0 = codes_to_16<FC_F16>(vx[t].x, vx[t].y), v1 = codes_to_16<FC_F16>(vx[t].z, vx[t].w);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                o[mt][t] = mfma16<FC_F16>(v0, p[mt][0], o[mt][t]);
                o[mt][t] = mfma16<FC_F16>(v1, p[mt][1], o[mt][t]);
            }
        }
    }

    // the waves' parts through LDS
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = wave * kRows + 16 * mt + col;
        const float sum = row_sum(l[mt]);
        if (quarter == 0) {
            lds_m[r] = m[mt];
            lds_l[r] = sum;
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
            *reinterpret_cast<f32x4_t *>(lds_o + r * kPitch + 16 * t + 4 * quarter) = o[mt][t] * unit_v;
    }
    __syncthreads();
    constexpr int kPieces = DP / 4;
    const int64_t part = ((((int64_t)b * g.kv_heads + h) * a.tiles + tile) * a.splits + split) * kRows;
    for (int i = threadIdx.x; i < rows * kPieces; i += kThreads) {
        const int r = i / kPieces, c = i % kPieces * 4;
        float most = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, lds_m[w * kRows + r]);
        const float base = most == -__builtin_inff() ? 0.f : most;
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds_m[w * kRows + r] - base);
            total += f * lds_l[w * kRows + r];
            sum += f * *reinterpret_cast<const f32x4_t *>(lds_o + (w * kRows + r) * kPitch + c);
        }
        if (active > 1) {
            *reinterpret_cast<f32x4_t *>(a.part_out + (part + r) * DP + c) = sum;
            if (c == 0) a.part_ml[part + r] = make_float2(most, total);
            continue;
        }
        const int q = (int)fast_div((uint32_t)(head0 + r), a.div_group);
        const int64_t row = ((int64_t)(s.row0 + token0 + (LIST ? 0 : q)) * a.heads + h * a.group + head0 + r - (LIST ? 0 : q * a.group));
        finish_row<DT>(a, row, c, sum, most, total);
    }
}

// The pieces of a row: a workgroup takes one row, its threads four channels each of every (kThreads / (DP / 4))-th piece.
template <int DT, int DP> __global__ __launch_bounds__(kThreads) void k_attend_join(AttnArgs a, int rows_tile, int list)
{
    constexpr int kPieces = DP / 4, kSets = kThreads / kPieces;
    __shared__ f32x4_t sums[kSets][kPieces];
    __shared__ float totals[kSets];
    const KvGeom &g = a.kv;
    uint32_t at = blockIdx.x;
    const int r = at % rows_tile;
    at /= rows_tile;
    const int tile = at % a.tiles;
    at /= a.tiles;
    const int h = at % g.kv_heads, b = at / g.kv_heads;
    const Sequence s = sequence_of(g, b);
    int token, head, token_last;
    if (list) {
        const int per_token = (a.group + rows_tile - 1) / rows_tile;
        token_last = token = tile / per_token;
        head = tile % per_token * rows_tile + r;
        if (head >= a.group) return;
    } else {
        const int row = tile * rows_tile + r;
        token = (int)fast_div((uint32_t)row, a.div_group);
        head = row - token * a.group;
        token_last = (int)fast_div((uint32_t)(min(tile * rows_tile + rows_tile, s.n * a.group) - 1), a.div_group);
    }
    if (token >= s.n) return;
    const int last = a.causal ? s.pos0 + token_last : s.len - 1;
    int blocks = last < 0 ? 0 : last / kBlock + 1;
    if (list) blocks = min(blocks, a.selected_width);
    const int active = max((blocks + a.per_split - 1) / a.per_split, 1);
    if (active == 1) return;        // (written whole)
    const int64_t part = ((((int64_t)b * g.kv_heads + h) * a.tiles + tile) * a.splits) * rows_tile + r;
    const int c = threadIdx.x % kPieces, set = threadIdx.x / kPieces;
    float most = -__builtin_inff();
    for (int i = threadIdx.x & 63; i < active; i += 64) most = fmaxf(most, a.part_ml[part + (int64_t)i * rows_tile].x);
#pragma unroll
    for (int i = 32; i; i >>= 1) most = fmaxf(most, __shfl_xor(most, i));
    const float base = most == -__builtin_inff() ? 0.f : most;
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    if (set < kSets)
        for (int i = set; i < active; i += kSets) {
            const float2 ml = a.part_ml[part + (int64_t)i * rows_tile];
            const float f = __builtin_amdgcn_exp2f(ml.x - base);
            total += f * ml.y;
            sum += f * *reinterpret_cast<const f32x4_t *>(a.part_out + (part + (int64_t)i * rows_tile) * DP + 4 * c);
        }
    if (set < kSets) {
        sums[set][c] = sum;
        if (c == 0) totals[set] = total;
    }
    __syncthreads();
    if (set) return;
    for (int i = 1; i < kSets; ++i) {
        sum += sums[i][c];
        total += totals[i];
    }
    finish_row<DT>(a, (int64_t)(s.row0 + token) * a.heads + h * a.group + head, 4 * c, sum, most, total);
}

template <int DT, int DP> hipError_t run_join(const AttnArgs &a, int rows_tile, bool list, hipStream_t s)
{
    const int64_t units = (int64_t)a.kv.batch * a.kv.kv_heads * a.tiles;
    k_attend_join<DT, DP><<<dim3((uint32_t)(units * rows_tile)), kThreads, 0, s>>>(a, rows_tile, list);
    return hipGetLastError();
}

template <int DT, int DP, int MT, bool LIST> hipError_t run_rows(const AttnArgs &a, hipStream_t s)
{
    constexpr size_t lds = (size_t)kWaves * 16 * MT * (DP + 4 + 2) * sizeof(float);
    if (lds > 64 * 1024) {
        const hipError_t e = raise_lds<k_attend_rows<DT, DP, MT, LIST>>(lds);
        if (e != hipSuccess) return e;
    }
    const int64_t units = (int64_t)a.kv.batch * a.kv.kv_heads * a.tiles;
    k_attend_rows<DT, DP, MT, LIST><<<dim3((uint32_t)(units * a.splits)), kThreads, lds, s>>>(a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || a.splits == 1 ? e : run_join<DT, DP>(a, 16 * MT, LIST, s);
}

template <int DT, int DP> hipError_t run_dim(const AttnArgs &a, int rows_tile, hipStream_t s)
{
    if (a.selected) return run_rows<DT, DP, 1, true>(a, s);
    if constexpr (DP <= 128)
        if (rows_tile == 32) return run_rows<DT, DP, 2, false>(a, s);
    return run_rows<DT, DP, 1, false>(a, s);
}

template <int DT> hipError_t run_type(const AttnArgs &a, int rows_tile, hipStream_t s)
{
    switch (a.kv.dp) {
    case 64: return run_dim<DT, 64>(a, rows_tile, s);
    case 128: return run_dim<DT, 128>(a, rows_tile, s);
    case 192: return run_dim<DT, 192>(a, rows_tile, s);
    default: return run_dim<DT, 256>(a, rows_tile, s);
    }
}

template <int DT> hipError_t join_type(const AttnArgs &a, int rows_tile, bool list, hipStream_t s)
{
    switch (a.kv.dp) {
    case 64: return run_join<DT, 64>(a, rows_tile, list, s);
    case 128: return run_join<DT, 128>(a, rows_tile, list, s);
    case 192: return run_join<DT, 192>(a, rows_tile, list, s);
    default: return run_join<DT, 256>(a, rows_tile, list, s);
    }
}

} // namespace

hipError_t launch_attend_join(const AttnArgs &a, int dtype, int rows_tile, bool list, hipStream_t s)
{
    return dtype == FC_BF16 ? join_type<FC_BF16>(a, rows_tile, list, s) : join_type<FC_F16>(a, rows_tile, list, s);
}

hipError_t launch_attend_rows(const AttnArgs &a, int dtype, int rows_tile, hipStream_t s)
{
    return dtype == FC_BF16 ? run_type<FC_BF16>(a, rows_tile, s) : run_type<FC_F16>(a, rows_tile, s);
}

} // namespace fc
