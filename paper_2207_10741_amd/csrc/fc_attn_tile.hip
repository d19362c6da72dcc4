// Attention of many rows: prompts and pieces of them.
//
// A workgroup holds 32 rows a wave (new tokens x the heads of one key head's group) and goes over the sequence's blocks.  A block's codes
// become 16-bit floats once, on their way into LDS, where all waves read them as operands; the next block's codes are in
// registers meanwhile.  S^T = K q^T with v_mfma_f32_32x32x16: a lane holds 32 scores of one row, so the softmax is the lane's own but for one
// exchange between the halves of the wave, and its weights are the other product's operand as they are (fc_attn_internal.hpp).
// The vector unit's work for a score is a multiply-add, an exponential, half a maximum, an addition and half a conversion.
#include "fc_attn_internal.hpp"

namespace fc {

namespace {

constexpr int kThreads = 2 * kTileRows;
template <int DT> __device__ __forceinline__ f32x16_t mfma_32(const uint4 &a, const uint4 &b, const f32x16_t &c) { return mfma32<DT>(a, b, c); }

template <int DP> constexpr uint32_t kKeyPitch = 2 * DP + 16;
constexpr uint32_t kValuePitch = 2 * kBlock + 16;

template <int DT, int DP> __global__ __launch_bounds__(kThreads, DP <= 128 ? 2 : 1) void k_attend_tile(AttnArgs a)
{
    constexpr int kRows = kTileRows, kSteps = DP / 16, kOut = DP / 32;
    constexpr int kShare = 4 * DP / kThreads;       // 16-byte pieces of the codes of keys (values) a thread brings
    // rows of keys and values in LDS; the 16 bytes behind each put rows that are read together into different banks
    constexpr uint32_t kKeyRow = kKeyPitch<DP>, kKeys = kBlock * kKeyRow, kValueRow = kValuePitch, kBuffer = kKeys + DP * kValueRow;
    extern __shared__ __align__(16) unsigned char lds[];
    const KvGeom &g = a.kv;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;

    // key heads of sequences first, so that a head's tiles run on one XCD where their number is a multiple of eight; long tiles first
    const int units = g.batch * g.kv_heads;
    uint32_t at = blockIdx.x;
    const int unit_rows = at % units;
    at /= units;
    const int split = at % a.splits, tile = a.tiles - 1 - (int)(at / a.splits);
    const int h = unit_rows % g.kv_heads, b = unit_rows / g.kv_heads;
    const Sequence s = sequence_of(g, b);
    const int rows = min(max(s.n * a.group - tile * kRows, 0), kRows);
    if (rows == 0) return;
    const int r = tile * kRows + wave * 32 + col;
    const bool valid = wave * 32 + col < rows;
    const int token = row_place(a, r).token;
    const int last = valid ? (a.causal ? s.pos0 + token : s.len - 1) : -1;
    const int token_last = (int)fast_div((uint32_t)(tile * kRows + rows - 1), a.div_group);
    const int last_most = a.causal ? s.pos0 + token_last : s.len - 1;
    // the wave's own bounds
    const int wave_rows = min(max(rows - wave * 32, 0), 32);
    const int wave_first = a.causal ? s.pos0 + (int)fast_div((uint32_t)(tile * kRows + wave * 32), a.div_group) : s.len - 1;
    const int wave_last = wave_rows == 0 ? -1 : a.causal ? s.pos0 + (int)fast_div((uint32_t)(tile * kRows + wave * 32 + wave_rows - 1), a.div_group) : s.len - 1;
    const int blocks = last_most < 0 ? 0 : last_most / kBlock + 1;
    const int active = max((blocks + a.per_split - 1) / a.per_split, 1);
    if (split >= active) return;
    const int begin = split * a.per_split, end = min(blocks, begin + a.per_split);

    uint4 q[kSteps];
    {
        // (rows behind the last repeat it and are left out below)
        const RowPlace p = row_place(a, min(r, tile * kRows + rows - 1));
        const uint16_t *const row = a.q + (s.row0 + p.token) * a.q_row + (int64_t)(h * a.group + p.head) * a.q_head;
        if (a.wide) {
#pragma unroll
            for (int c = 0; c < kSteps; ++c) q[c] = flip_signs(load8<true>(row, 16 * c + 8 * half, g.d), a.signs);
        } else {
#pragma unroll
            for (int c = 0; c < kSteps; ++c) q[c] = flip_signs(load8<false>(row, 16 * c + 8 * half, g.d), a.signs);
        }
    }

    f32x16_t o[kOut];
#pragma unroll
    for (int t = 0; t < kOut; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -__builtin_inff(), l = 0.f, unit_v = 1.f;     // m: the row's weights are 2^(z - m)

    uint4 kx[kShare], vx[kShare];
    float2 scales;
    bool there;
    auto bring = [&](int block) {
        const int32_t pool = pool_block(g, b, block);
        there = pool >= 0;
        const int64_t unit = unit_of(g, max(pool, 0), h);
        const uint8_t *const from = g.codes + unit * (2 * kBlock * DP);
        scales = g.scales[unit];
#pragma unroll
        for (int i = 0; i < kShare; ++i) {
            kx[i] = *reinterpret_cast<const uint4 *>(from + i * kThreads * 16 + threadIdx.x * 16u);
            vx[i] = *reinterpret_cast<const uint4 *>(from + (4 * DP + i * kThreads) * 16 + threadIdx.x * 16u);
        }
    };
    if (begin < end) bring(begin);
    // where the thread's first pieces go and where the lane's operands are, from the buffer's start on
    auto key_place = [](uint32_t piece) {       // (see key_piece)
        const uint32_t channel = (piece >> 6) % (DP / 64) * 64 + (piece >> 4 & 3) * 16, token = (piece >> 6) / (DP / 64) * 16 + (piece & 15);
        return token * kKeyRow + channel * 2;
    };
    const uint32_t key_to = key_place(threadIdx.x);
    // four words of four tokens 16 w + 4 quarter .. + 3: as the scores' lanes hold them, half `quarter & 1`
    const uint32_t value_to = kKeys + ((threadIdx.x >> 6) * 16 + (threadIdx.x & 15)) * kValueRow + (threadIdx.x >> 4 & 1) * 16 + (threadIdx.x >> 5 & 1) * 8;
    const uint32_t key_at = col * kKeyRow + half * 16, value_at = kKeys + col * kValueRow + half * 16;
    uint32_t buffer = 0;
    for (int block = begin; block < end; ++block, buffer = kBuffer - buffer) {
        const bool here = there;
        const float scale_k = here ? scales.x : 1.f, scale_v = here ? __builtin_fabsf(scales.y) : unit_v;
        const bool strange = here && scales.y < 0.f;        // (NaN among the values: zeros in LDS, found again below)
        if (!keeps_unit(scale_v, unit_v)) {
            const float factor = pow2_ratio(unit_v, scale_v);
#pragma unroll
            for (int t = 0; t < kOut; ++t) o[t] *= factor;
            unit_v = scale_v;
        }
        const float to_unit = pow2_ratio(scale_v, unit_v);
        unsigned char *const keys_to = lds + buffer + key_to, *const values_to = lds + buffer + value_to;
        const unsigned char *const keys = lds + buffer + key_at, *const values = lds + buffer + value_at;
#pragma unroll
        for (int i = 0; i < kShare; ++i) {
            // (kThreads pieces further; a constant unless they split a token's channels)
            constexpr uint32_t kValueStep = kThreads / 4 * kValueRow;
            const uint32_t key_step = DP % 192 ? key_place(i * kThreads) : key_place(threadIdx.x + i * kThreads) - key_to;
            *reinterpret_cast<uint4 *>(keys_to + key_step) = codes_to_16<DT>(kx[i].x, kx[i].y);
            *reinterpret_cast<uint4 *>(keys_to + key_step + 16) = codes_to_16<DT>(kx[i].z, kx[i].w);
            if (strange) vx[i] = without_nan(vx[i]);
            const uint4 first = codes_to_f16(vx[i].x, vx[i].y, to_unit), second = codes_to_f16(vx[i].z, vx[i].w, to_unit);
            const uint2 words[4] = {make_uint2(first.x, first.y), make_uint2(first.z, first.w), make_uint2(second.x, second.y), make_uint2(second.z, second.w)};
#pragma unroll
            for (int w = 0; w < 4; ++w) *reinterpret_cast<uint2 *>(values_to + i * kValueStep + 32 * w) = words[w];
        }
        __syncthreads();
        if (block + 1 < end) bring(block + 1);
        if (!here || block * kBlock > wave_last) continue;

        f32x16_t z[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[t][i] = 0.f;
#pragma unroll
            for (int c = 0; c < kSteps; ++c)
                z[t] = mfma_32<DT>(*reinterpret_cast<const uint4 *>(keys + 32 * t * kKeyRow + 32 * c), q[c], z[t]);
        }

        float to_log2 = a.scale_log2 * scale_k;
        const bool partly = block * kBlock + kBlock - 1 > wave_first;
        const int left = last - block * kBlock - 4 * half;      // scores i of tile t whose token 32 t + 8 (i / 4) + i % 4 is at most this are seen
        if (partly) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[t][i] = 32 * t + 8 * (i >> 2) + (i & 3) <= left ? z[t][i] * to_log2 : -__builtin_inff();
            to_log2 = 1.f;      // (a factor of zero would make NaN of what is masked)
        }
        float most = z[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) most = fmaxf(most, z[i >> 4][i & 15]);
        most = max_over_32(most) * to_log2;
        if (__any(most - m > kSlack)) {
            const float m_new = fmaxf(m, most);
            const float factor = m_new == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= factor;
#pragma unroll
            for (int t = 0; t < kOut; ++t) o[t] *= factor;
        }
        const float base = m == -__builtin_inff() ? 0.f : -m;
        uint4 p[4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][i], to_log2, base));
                const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][i + 1], to_log2, base));
                l += e0;
                l += e1;
                w[i >> 1] = pack2<FC_F16>(e0, e1);
            }
            p[2 * t] = make_uint4(w[0], w[1], w[2], w[3]);
            p[2 * t + 1] = make_uint4(w[4], w[5], w[6], w[7]);
        }

#pragma unroll
        for (int t = 0; t < kOut; ++t)
#pragma unroll
            for (int step = 0; step < 4; ++step)
                o[t] = mfma_32<FC_F16>(*reinterpret_cast<const uint4 *>(values + 32 * t * kValueRow + 32 * step), p[step], o[t]);
        if (strange) {
            const uint8_t *const codes = g.codes + unit_of(g, max(pool_block(g, b, block), 0), h) * (2 * kBlock * DP);
#pragma unroll
            for (int t = 0; t < kOut; ++t) {
                f32x16_t count;
#pragma unroll
                for (int i = 0; i < 16; ++i) count[i] = 0.f;
#pragma unroll
                for (int step = 0; step < 4; ++step) {
                    // tokens 16 step + 4 half + 0 .. 3 and 8 on: quarters `half` and half + 2 of the row
                    const uint32_t lo = *reinterpret_cast<const uint32_t *>(codes + value_piece<DP>(32 * t + col, 16 * half) + 4 * step);
                    const uint32_t hi = *reinterpret_cast<const uint32_t *>(codes + value_piece<DP>(32 * t + col, 16 * (half + 2)) + 4 * step);
                    const uint4 seen = make_uint4(seen_pair(16 * step, left), seen_pair(16 * step + 2, left), seen_pair(16 * step + 8, left),
                                                  seen_pair(16 * step + 10, left));
                    count = mfma_32<FC_F16>(nan_marks(lo, hi), seen, count);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] = count[i] > 0.f ? __builtin_nanf("") : o[t][i];
            }
        }
    }

    l += __shfl_xor(l, 32);
    const int64_t unit = (int64_t)unit_rows * a.tiles + tile;
    const Pieces<DP> pieces(a, unit, kRows);
    auto out_row = [&](int row) {
        const RowPlace p = row_place(a, tile * kRows + row);
        return (int64_t)(s.row0 + p.token) * a.heads + h * a.group + p.head;
    };
    if (valid) {
        const int64_t row = out_row(wave * 32 + col);
        const uint32_t part = (uint32_t)(split * kRows + wave * 32 + col);
        if (active > 1 && half == 0) pieces.put_ml(part, m, l);
#pragma unroll
        for (int t = 0; t < kOut; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int c = 32 * t + 2 * i + 4 * half;
                const f32x4_t v = {o[t][i] * unit_v, o[t][i + 1] * unit_v, o[t][i + 2] * unit_v, o[t][i + 3] * unit_v};
                if (active > 1) pieces.put(part, c, v);
                else finish_row<DT>(a, row, c, v, m, l);
            }
    }
    if (active == 1) return;
    __syncthreads();        // (the flag lies where operands were)
    if (!last_to_arrive(a, unit, active, reinterpret_cast<int32_t *>(lds))) return;
    join_pieces<DT, DP, kThreads>(a, pieces, rows, kRows, active, reinterpret_cast<float *>(lds) + 4, out_row);
}

template <int DT, int DP> hipError_t run_tile(const AttnArgs &a, hipStream_t s)
{
    constexpr size_t lds = 2 * (size_t)(kBlock * kKeyPitch<DP> + DP * kValuePitch);
    const hipError_t raised = raise_lds<k_attend_tile<DT, DP>>(lds);
    if (raised != hipSuccess) return raised;
    const int64_t units = (int64_t)a.kv.batch * a.kv.kv_heads * a.tiles;
    k_attend_tile<DT, DP><<<dim3((uint32_t)(units * a.splits)), kThreads, lds, s>>>(a);
    return hipGetLastError();
}

template <int DT> hipError_t run_type(const AttnArgs &a, hipStream_t s)
{
    switch (a.kv.dp) {
    case 64: return run_tile<DT, 64>(a, s);
    case 128: return run_tile<DT, 128>(a, s);
    case 192: return run_tile<DT, 192>(a, s);
    default: return run_tile<DT, 256>(a, s);
    }
}

} // namespace

hipError_t launch_attend_tile(const AttnArgs &a, int dtype, hipStream_t s)
{
    return dtype == FC_BF16 ? run_type<FC_BF16>(a, s) : run_type<FC_F16>(a, s);
}

} // namespace fc
