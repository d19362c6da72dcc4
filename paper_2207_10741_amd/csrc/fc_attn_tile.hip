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

template <int DT> __device__ __forceinline__ f32x16_t mfma_32(const uint4 &a, const uint4 &b, const f32x16_t &c) { return mfma32<DT>(a, b, c); }

constexpr int kAhead = 4;
template <int DP> constexpr uint32_t kKeyPitch = 2 * DP + 16;
constexpr uint32_t kValuePitch = 2 * kBlock + 16;

// 32 rows a wave: scores, weights and outputs of 64 would not fit the registers without copies between their halves (820 us against 573).  A step multiplies a
// block's values with the last step's weights beside this step's scores, so that the matrix cores always have the one while the vector unit works on the other.
// 8192 tokens, 32 heads of 128 over 8, causal: 538 - 557 us, 990 - 1020 TFLOP/s, 86 - 89 % of what the library's 8192^3 product reaches here.  Bound by the matrix cores, and then by power
// (the clock falls as their share of idle cycles does).
template <int DT, int DP, int WAVES> __global__ __launch_bounds__(64 * WAVES, DP <= 128 ? 2 : 1) void k_attend_tile(AttnArgs a)
{
    constexpr int kWaves = WAVES, kThreads = 64 * kWaves, kRows = 32 * kWaves, kSteps = DP / 16, kOut = DP / 32;
    constexpr int kShare = (4 * DP + kThreads - 1) / kThreads;      // 16-byte pieces of the codes of keys (values) a thread brings
    constexpr bool kEven = 4 * DP % kThreads == 0;                  // (every thread; else the last ones are some waves')
    // rows of keys and values in LDS; the 16 bytes behind each put rows that are read together into different banks
    constexpr uint32_t kKeyRow = kKeyPitch<DP>, kValues = kBlock * kKeyRow, kValueRow = kValuePitch, kBuffer = kValues + DP * kValueRow;
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
    const int r = wave * 32 + col;      // the lane's row, and the last position that it attends to
    const int last = r < rows ? (a.causal ? s.pos0 + row_place(a, tile * kRows + r).token : s.len - 1) : -1;
    const int token_last = (int)fast_div((uint32_t)(tile * kRows + rows - 1), a.div_group);
    const int last_most = a.causal ? s.pos0 + token_last : s.len - 1;
    const int wave_first = a.causal ? s.pos0 + row_place(a, tile * kRows + wave * 32).token : s.len - 1;     // the least `last` of the wave's rows
    const int blocks = last_most < 0 ? 0 : last_most / kBlock + 1;
    const int active = max((blocks + a.per_split - 1) / a.per_split, 1);
    if (split >= active) return;
    const int begin = split * a.per_split, end = min(blocks, begin + a.per_split);

    uint4 q[kSteps];
    {
        // (rows behind the last repeat it and are left out below)
        const RowPlace at_row = row_place(a, tile * kRows + min(r, rows - 1));
        const uint16_t *const row = a.q + (s.row0 + at_row.token) * a.q_row + (int64_t)(h * a.group + at_row.head) * a.q_head;
        if (a.wide) {
#pragma unroll
            for (int c = 0; c < kSteps; ++c) q[c] = flip_signs(load8<true>(row, 16 * c + 8 * half, g.d), a.signs);
        } else {
#pragma unroll
            for (int c = 0; c < kSteps; ++c) q[c] = flip_signs(load8<false>(row, 16 * c + 8 * half, g.d), a.signs);
        }
    }

    // what a row holds: o in its unit, weights 2^(z - m), m a whole number, l this lane's part of their sum
    f32x16_t o[kOut], z;
    float m = -__builtin_inff(), l = 0.f;
    RunningUnit o_unit;
    o_unit.clear();
    uint4 p[2];     // weights of the last half-block whose product with the values is still to come
#pragma unroll
    for (int t = 0; t < kOut; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    p[0] = p[1] = make_uint4(0, 0, 0, 0);

    // where the thread's first pieces go and where the lane's operands are, from a buffer's start on
    auto key_place = [](uint32_t piece, uint32_t n) {
        const KeyHalf k = key_half<DP>(piece, n);
        return k.token * kKeyRow + k.channel * 2;
    };
    const uint32_t key_to = key_place(threadIdx.x, 0);
    // four words of four tokens 16 w + 4 quarter .. + 3: as the scores' lanes hold them, half `quarter & 1`
    const uint32_t value_to = kValues + ((threadIdx.x >> 6) * 16 + (threadIdx.x & 15)) * kValueRow + (threadIdx.x >> 4 & 1) * 16 + (threadIdx.x >> 5 & 1) * 8;
    const uint32_t key_at = col * kKeyRow + half * 16, value_at = kValues + col * kValueRow + half * 16;

    // A block's codes on their way: global memory -> registers -> LDS, as 16-bit floats.
    uint4 kx[kShare], vx[kShare];
    auto codes_of = [&](int32_t pool) { return g.codes + unit_of(g, max(pool, 0), h) * (2 * kBlock * DP); };
    auto bring = [&](const uint8_t *from, uint4 (&x)[kShare]) {
#pragma unroll
        for (int i = 0; i < kShare; ++i)
            if (kEven || i * kThreads + (int)threadIdx.x < 4 * DP) x[i] = *reinterpret_cast<const uint4 *>(from + i * kThreads * 16 + threadIdx.x * 16u);
    };
    // (kThreads pieces further: a constant unless they split a token's channels)
    auto key_step = [&](int i, int n) { return DP % 96 ? key_place(i * kThreads, n) : key_place(threadIdx.x + i * kThreads, n) - key_to; };
    // half a piece of keys (16 bytes in LDS) and of values (two words of four tokens)
    auto put_keys = [&](uint32_t buffer, int i, int n) {
        if (!kEven && i * kThreads + (int)threadIdx.x >= 4 * DP) return;
        *reinterpret_cast<uint4 *>(lds + buffer + key_to + key_step(i, n)) = n ? codes_to_16<DT>(kx[i].z, kx[i].w) : codes_to_16<DT>(kx[i].x, kx[i].y);
    };
    auto put_values = [&](uint32_t buffer, float to_unit, int i, int n) {
        if (!kEven && i * kThreads + (int)threadIdx.x >= 4 * DP) return;
        const uint4 x = n ? codes_to_f16(vx[i].z, vx[i].w, to_unit) : codes_to_f16(vx[i].x, vx[i].y, to_unit);
        unsigned char *const to = lds + buffer + value_to + i * (kThreads / 4 * kValueRow) + 64 * n;
        *reinterpret_cast<uint2 *>(to) = make_uint2(x.x, x.y);
        *reinterpret_cast<uint2 *>(to + 32) = make_uint2(x.z, x.w);
    };
    auto key_operand = [&](uint32_t buffer, int t, int c) { return *reinterpret_cast<const uint4 *>(lds + buffer + key_at + 32 * t * kKeyRow + 32 * c); };
    auto value_operand = [&](uint32_t buffer, int t, int step) {
        return *reinterpret_cast<const uint4 *>(lds + buffer + value_at + 32 * t * kValueRow + 32 * step);
    };

    // Half t (32 tokens) of a block: its scores z become weights, while the matrix cores make the next half's scores (from keys_next, half t ^ 1)
    // and add the last half's part to o (from values_last, weights p).  The two share no operand, so their instructions alternate.
    auto half_block = [&](auto t_const, int block, bool here, float to_log2, uint32_t keys_next, uint32_t values_last, auto beside) {
        constexpr int t = decltype(t_const)::value;
        const int from = block * kBlock + 32 * t;
        if (static_cast<int>(!here) | static_cast<int>(from + 31 > wave_first)) {       // (one branch: two take 1.5 % longer on long prompts)
            const int left = here ? last - from - 4 * half : -1;        // scores i whose token 8 (i / 4) + i % 4 is at most this are seen
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 8 * (i >> 2) + (i & 3) <= left ? z[i] * to_log2 : -__builtin_inff();
            to_log2 = 1.f;      // (a factor of zero would make NaN of what is masked)
        }
        float most = z[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = fmaxf(most, z[i]);
        most = max_over_32(most) * to_log2;
        if (__any(most - m > kSlack)) {
            const float m_new = fmaxf(m, __builtin_ceilf(most) - kLead);
            const float factor = m_new == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - m_new);     // (a power of two: nothing is rounded)
            m = m_new;
            l *= factor;
#pragma unroll
            for (int i = 0; i < kOut; ++i) o[i] *= factor;
            const f16x2_t two = __builtin_bit_cast(f16x2_t, pack2<FC_F16>(factor, factor));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t w[4] = {p[i].x, p[i].y, p[i].z, p[i].w};
                uint32_t r[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, w[j]) * two);
                p[i] = make_uint4(r[0], r[1], r[2], r[3]);
            }
        }
        const float base = m == -__builtin_inff() ? 0.f : -m;
        f32x16_t z_next;
#pragma unroll
        for (int i = 0; i < 16; ++i) z_next[i] = 0.f;
        // Step by step, in this order: matrix instructions on one operand from LDS, the operand of one kAhead steps on, and the vector unit's work of that time.
        constexpr int kProducts = 2 * kSteps;
        auto operand = [&](int i) {
            return i % 2 == 0 ? key_operand(keys_next, t ^ 1, i / 2) : value_operand(values_last, i / 2 % kOut, 2 * (t ^ 1) + i / 2 / kOut);
        };
        uint4 x[kProducts];
        uint32_t w[8];
        float e[16];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) x[i] = operand(i);
#pragma unroll
        for (int i = 0; i < kProducts; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i + kAhead < kProducts) x[i + kAhead] = operand(i + kAhead);
            if (i % 2 == 0) z_next = mfma_32<DT>(x[i], q[i / 2], z_next);
            else o[i / 2 % kOut] = mfma_32<FC_F16>(x[i], p[i / 2 / kOut], o[i / 2 % kOut]);
#pragma unroll
            for (int j = 16 * i / kProducts; j < 16 * (i + 1) / kProducts; ++j) {
                e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j], to_log2, base));
                l += e[j];
                if (j & 1) {
                    w[j >> 1] = pack2<FC_F16>(e[j - 1], e[j]);
                    __asm__ volatile("" : "+v"(w[j >> 1]), "+v"(l));     // (here, not where it is used)
                }
            }
            // (late: what it works on has then been on its way for longer than a half)
            constexpr int kLate = kProducts / 2, kBeside = 4 * kShare;
#pragma unroll
            for (int n = ((i - kLate) * kBeside + kLate - 1) / kLate; i >= kLate && n < ((i + 1 - kLate) * kBeside + kLate - 1) / kLate; ++n) beside(n);
        }
        __builtin_amdgcn_sched_barrier(0);
        p[0] = make_uint4(w[0], w[1], w[2], w[3]);
        p[1] = make_uint4(w[4], w[5], w[6], w[7]);
        z = z_next;
    };

    // What half t of a block adds to o (weights p), its values taken from memory: exact products in units of its scale, added to o in 32 bits.
    auto far_values = [&](int32_t pool, int t, int to_unit) {
        uint32_t at = value_piece<DP>(col, 16 * half) + 8 * t;
        __asm__ volatile("" : "+v"(at));        // (made here, not kept in a register all along)
        const uint8_t *const from = codes_of(pool) + at;
        const float ratio = pow2_held(to_unit);
#pragma unroll
        for (int n = 0; n < kOut; ++n) {
            f32x16_t adds;
            __builtin_amdgcn_sched_barrier(0);      // (one after another, in few registers)
#pragma unroll
            for (int i = 0; i < 16; ++i) adds[i] = 0.f;
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                // tokens 16 (2 t + step) + 4 half + 0 .. 3 and 8 on: quarters `half` and half + 2 of the row
                uint32_t lo = *reinterpret_cast<const uint32_t *>(from + value_piece<DP>(32 * n, 0) - value_piece<DP>(0, 0) + 4 * step);
                uint32_t hi = *reinterpret_cast<const uint32_t *>(from + value_piece<DP>(32 * n, 32) - value_piece<DP>(0, 0) + 4 * step);
                adds = mfma_32<FC_F16>(codes_to_16<FC_F16>(lo & ~nan_bytes(lo), hi & ~nan_bytes(hi)), p[step], adds);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) o[n][i] = __builtin_fmaf(adds[i], ratio, o[n][i]);
        }
    };

    if (begin < end) {
        // Block j's first half runs with keys of j and values of j - 1 in LDS, its second with keys of j + 1 and values of j.  These are put there beside the
        // first half, so that a barrier between the halves is the only one; both are brought to registers beside the second half before.
        // Lane i holds where the i-th of 64 blocks is in the pool and its scales (two blocks ahead of the loop): no scalar load in the loop, behind which the
        // waits for LDS would be waits for all of it.
        int32_t held_pool = -1;
        float2 held_scales = make_float2(1.f, 1.f);
        auto look_up = [&](int first) {
            held_pool = -1;
            if (first + lane < end) {
                held_pool = pool_block(g, b, first + lane);
                held_scales = g.scales[unit_of(g, max(held_pool, 0), h)];
            }
            __asm__ volatile("" : "+v"(held_pool), "+v"(held_scales.x), "+v"(held_scales.y));      // (waited for here)
        };
        auto pool_at = [&](int i) { return __builtin_amdgcn_readlane(held_pool, i & 63); };
        auto scales_at = [&](int i) {
            return make_float2(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_scales.x), i & 63)),
                               __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_scales.y), i & 63)));
        };
        look_up(begin);
        int32_t pool = pool_at(0), pool_next = pool_at(1);
        float2 scales = scales_at(0), scales_next = scales_at(1);
        bring(codes_of(pool), kx);
#pragma unroll
        for (int i = 0; i < 2 * kShare; ++i) put_keys(0, i / 2, i % 2);
        bring(codes_of(pool_next), kx);
        bring(codes_of(pool) + kBlock * DP, vx);
        for (uint32_t i = threadIdx.x * 16; i < DP * kValueRow; i += kThreads * 16)      // (values before the first: finite, for weights of zero)
            *reinterpret_cast<uint4 *>(lds + kBuffer + kValues + i) = make_uint4(0, 0, 0, 0);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kSteps; ++c) z = mfma_32<DT>(key_operand(0, 0, c), q[c], z);

        uint32_t buffer = 0;        // of block j's keys and values; the other one is its neighbours'
        for (int block = begin; block < end; ++block, buffer = kBuffer - buffer) {
            const bool here = pool >= 0;
            const float to_log2 = here ? score_factor(a, scales.x) : 1.f;
            const bool strange = here && scales.y < 0.f;    // NaN among the values: zeros in LDS, found again here
            if (strange) {
                const uint8_t *const codes = codes_of(pool);
                const int left = last - block * kBlock - 4 * half;
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
#pragma unroll
                for (int i = 0; i < kShare; ++i) vx[i] = without_nan(vx[i]);
            }
            const int scale_v = here ? exponent_of(scales.y) : o_unit.e, unit_new = here ? o_unit.with(scale_v) : o_unit.e;
            const bool far = RunningUnit::far(scale_v, unit_new);       // values that f16 does not hold in the unit: zeros in LDS, and far_values
            const int32_t pool_far = pool;
            if (!here || far)
#pragma unroll
                for (int i = 0; i < kShare; ++i) vx[i] = make_uint4(0, 0, 0, 0);     // (finite, for weights of zero)
            const float to_unit = far ? 1.f : pow2_held(scale_v - unit_new);
            half_block(Const<0>(), block, here, to_log2, buffer, kBuffer - buffer, [&](int i) {
                if (i < 2 * kShare) put_keys(kBuffer - buffer, i / 2, i % 2);
                else put_values(buffer, to_unit, i / 2 - kShare, i % 2);
            });
            __syncthreads();

            if (unit_new != o_unit.e) {         // (o has all of the values that are in the old one)
                const float factor = pow2_held(o_unit.e - unit_new);
#pragma unroll
                for (int t = 0; t < kOut; ++t) o[t] *= factor;
                o_unit.e = unit_new;
            }
            if (__builtin_expect(far, 0)) far_values(pool_far, 0, scale_v - unit_new);
            pool = pool_next;
            scales = scales_next;
            if (block + 1 < end) bring(codes_of(pool) + kBlock * DP, vx);
            const int after = block + 2 - begin;        // (what is behind the end is not there)
            if (after % 64 == 0) look_up(block + 2);
            pool_next = pool_at(after);
            scales_next = scales_at(after);
            if (block + 2 < end) bring(codes_of(pool_next), kx);
            half_block(Const<1>(), block, here, to_log2, kBuffer - buffer, buffer, [](int) {});
            if (__builtin_expect(far, 0)) far_values(pool_far, 1, scale_v - unit_new);
        }
        // the last half's values
        buffer = kBuffer - buffer;
#pragma unroll
        for (int t = 0; t < kOut; ++t)
#pragma unroll
            for (int step = 0; step < 2; ++step) o[t] = mfma_32<FC_F16>(value_operand(buffer, t, 2 + step), p[step], o[t]);
    }

    const float to_sums = o_unit.to_sums();
    const int64_t unit = (int64_t)unit_rows * a.tiles + tile;
    const Pieces<DP> pieces(a, unit, kRows);
    auto out_row = [&](int row) {
        const RowPlace p = row_place(a, tile * kRows + row);
        return (int64_t)(s.row0 + p.token) * a.heads + h * a.group + p.head;
    };
    // Pieces are written as the registers hold them, 1 KB a store: [wave][output tile][four channels][lane].
    constexpr int kLanes = kOut * 4 * 64;
    auto place = [&](int item) {
        const int tile_at = item / kLanes, in = item % kLanes, row = tile_at * 32 + (in & 31);
        return ItemPlace{row < rows ? row : kNoRow, (in >> 8) * 32 + (in >> 6 & 3) * 8 + (in >> 5 & 1) * 4};
    };
    const float sum = l + __shfl_xor(l, 32);
    const int64_t row = out_row(min(r, rows - 1));
    if (active > 1 && half == 0) pieces.put_ml((uint32_t)(split * kRows + r), m, sum);
    const uint32_t item = (uint32_t)(split * kRows * (DP / 4) + wave * kLanes + lane);
#pragma unroll
    for (int t = 0; t < kOut; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const f32x4_t v = {o[t][i] * to_sums, o[t][i + 1] * to_sums, o[t][i + 2] * to_sums, o[t][i + 3] * to_sums};
            if (active > 1) pieces.put(item + (t * 4 + i / 4) * 64, v);
            else if (r < rows) finish_row<DT>(a, row, 32 * t + 2 * i + 4 * half, v, m, sum);
        }
    if (active == 1) return;
    __syncthreads();        // (the flag lies where operands were)
    if (!last_to_arrive(a, unit, active, reinterpret_cast<int32_t *>(lds))) return;
    join_pieces<DT, DP, kThreads>(a, pieces, (rows + 31) / 32 * kLanes, kRows, active, reinterpret_cast<float *>(lds) + 4, place, out_row);
}

template <int DT, int DP, int WAVES> hipError_t run_tile(const AttnArgs &a, hipStream_t s)
{
    constexpr size_t lds = 2 * (size_t)(kBlock * kKeyPitch<DP> + DP * kValuePitch);
    const hipError_t raised = raise_lds<k_attend_tile<DT, DP, WAVES>>(lds);
    if (raised != hipSuccess) return raised;
    const int64_t units = (int64_t)a.kv.batch * a.kv.kv_heads * a.tiles;
    k_attend_tile<DT, DP, WAVES><<<dim3((uint32_t)(units * a.splits)), 64 * WAVES, lds, s>>>(a);
    return hipGetLastError();
}

template <int DT> hipError_t run_type(const AttnArgs &a, int rows_tile, hipStream_t s)
{
    switch (a.kv.dp) {
    case 64: return run_tile<DT, 64, 4>(a, s);
    case 96: return rows_tile == 256 ? run_tile<DT, 96, 8>(a, s) : run_tile<DT, 96, 4>(a, s);
    case 128: return rows_tile == 256 ? run_tile<DT, 128, 8>(a, s) : run_tile<DT, 128, 4>(a, s);
    case 192: return run_tile<DT, 192, 4>(a, s);
    default: return run_tile<DT, 256, 4>(a, s);
    }
}

} // namespace

hipError_t launch_attend_tile(const AttnArgs &a, int dtype, int rows_tile, hipStream_t s)
{
    return dtype == FC_BF16 ? run_type<FC_BF16>(a, rows_tile, s) : run_type<FC_F16>(a, rows_tile, s);
}

} // namespace fc
