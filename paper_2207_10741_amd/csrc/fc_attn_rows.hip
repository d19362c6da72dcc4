// Attention of few rows over a long axis: single tokens, and tokens' lists of blocks.
//
// A wave holds 16 or 32 rows (new tokens x the heads of one key head's group) and goes over blocks with a softmax of its own.  A block goes
// from memory to registers in the order the matrix instructions want it (fc_attn_internal.hpp): no LDS, and no lane exchange but for the
// rows' maximum.  The next block's keys are on their way as soon as this one's are used, and its values likewise, so that a wave always has
// half a block in flight.
//   k_attend_rows: the waves of a workgroup take a piece's blocks of the sequence (or of a token's list) in turn and are joined through LDS; the last workgroup joins the pieces.
//   k_attend_lists: a wave takes a token's whole list.
//   k_attend_shared: a wave takes as many neighbouring tokens as fill its 16 rows, and every block that one of them has in its list once.
#include "fc_attn_internal.hpp"

namespace fc {

namespace {

// The blocks a wave goes over: the sequence's own, those of a list, or entries of several tokens' lists together (the block, and from bit 16 on a bit for every
// token that has it).
enum { kAllBlocks, kListed, kShared };

// A wave's rows and its running softmax.
template <int DT, int DP, int MT> struct Rows {
    static constexpr int kLoads = DP / 16, kTiles = DP / 16, kOperands = DP / 32;      // loads of a block's keys, of its values; instructions of 16 tokens' scores
    uint4 q[MT][kOperands];
    f32x4_t o[MT][kTiles];          // in its unit
    RunningUnit unit;
    float m[MT], l[MT];             // weights are 2^(z - m); l: this lane's part of their sum
    int last[MT];                   // the last position that the lane's row attends to
    int last_least;                 // ... of all rows
    uint32_t token, tokens;         // (kShared: the lane's token of the entries', and the bits of all)

    __device__ __forceinline__ void clear()
    {
        unit.clear();
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            m[mt] = -__builtin_inff();
            l[mt] = 0.f;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) o[mt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    }

    // The lane's row of tile mt.
    __device__ __forceinline__ void bring_queries(const AttnArgs &a, int mt, const uint16_t *row)
    {
        const int quarter = (threadIdx.x & 63) >> 4, d = a.kv.d;
        if (a.wide) {
#pragma unroll
            for (int c = 0; c < kOperands; ++c) q[mt][c] = flip_signs(load8<true>(row, channel_of(c, quarter), d), a.signs);
        } else {
#pragma unroll
            for (int c = 0; c < kOperands; ++c) q[mt][c] = flip_signs(load8<false>(row, channel_of(c, quarter), d), a.signs);
        }
    }

    // The first of the eight channels that the lane holds of operand c (key_at's order).
    __device__ static __forceinline__ int channel_of(int c, int quarter) { return DP == 96 && c == 2 ? 64 + quarter * 8 : (c >> 1) * 64 + quarter * 16 + (c & 1) * 8; }

    // Blocks first, first + step, ... below end of the sequence or of its list (both in order).
    template <int BLOCKS>
    __device__ __forceinline__ void run(const AttnArgs &a, int b, int h, const int32_t *__restrict__ list, int first, int step, int end)
    {
        const KvGeom &g = a.kv;
        if (first >= end) return;
        const int lane = threadIdx.x & 63, quarter = lane >> 4;
        // Lane i holds what the loop needs to know of its i-th block of 64 (of the list's blocks, where they are in the pool, their scales): the loop
        // itself waits for keys and values only.
        int held_block = 0, held_pool = -1;
        float2 held_scales = make_float2(1.f, 1.f);
        auto look_up = [&](int from) {
            const int j = from + lane * step;
            held_block = 0, held_pool = -1;
            if (j < end) {
                held_block = BLOCKS == kAllBlocks ? j : list[j];
                held_pool = pool_block(g, b, BLOCKS == kShared ? held_block & 0xffff : held_block);
                held_scales = g.scales[unit_of(g, max(held_pool, 0), h)];
            }
        };
        auto looked_up = [&] { __asm__ volatile("" : "+v"(held_block), "+v"(held_pool), "+v"(held_scales.x), "+v"(held_scales.y)); };    // (waited for there)
        look_up(first);
        int block = __builtin_amdgcn_readlane(held_block, 0), pool = __builtin_amdgcn_readlane(held_pool, 0);
        auto scales_at = [&](int i) {
            return make_float2(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_scales.x), i)),
                               __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(held_scales.y), i)));
        };
        // A block's codes: keys at 0, values behind them.  A block that is not there, and the one behind the last, is an empty buffer.
        auto codes_of = [&](int32_t p) {
            return __builtin_amdgcn_make_buffer_rsrc(g.codes + unit_of(g, max(p, 0), h) * (2 * kBlock * DP), 0, p < 0 ? 0 : 2 * kBlock * DP, 0x00020000);
        };
        uint4 kx[kLoads], vx[kTiles];
        auto bring_keys = [&](__amdgpu_buffer_rsrc_t from, int n) {
            kx[n] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(from, lane * 16, n * 1024, 0));
        };
        auto bring_values = [&](__amdgpu_buffer_rsrc_t from, int t) {
            vx[t] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(from, lane * 16, kBlock * DP + t * 1024, 0));
        };
        {
            const auto codes = codes_of(pool);
#pragma unroll
            for (int n = 0; n < kLoads; ++n) bring_keys(codes, n);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) bring_values(codes, t);
        }
        looked_up();
        float2 scales = scales_at(0);

        int i_next = 1;
        for (int j = first; j < end; j += step, ++i_next) {
            const bool more = j + step < end;
            if (i_next == 64 && more) {
                look_up(j + step);
                looked_up();
                i_next = 0;
            }
            const int block_next = __builtin_amdgcn_readlane(held_block, i_next & 63), pool_next = __builtin_amdgcn_readlane(held_pool, i_next & 63);
            const float2 scales_next = scales_at(i_next & 63);
            const bool here = pool >= 0;
            const auto codes_next = codes_of(more ? pool_next : -1);

            f32x4_t z[MT][4];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) z[mt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            auto scores = [&](int t, const uint4 &k, int c) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) z[mt][t] = mfma16<DT>(k, q[mt][c], z[mt][t]);
            };
            if constexpr (DP == 96) {
#pragma unroll
                for (int pair = 0; pair < 2; ++pair) {
                    scores(2 * pair, codes_to_16<DT>(kx[3 * pair].x, kx[3 * pair].y), 0);
                    scores(2 * pair, codes_to_16<DT>(kx[3 * pair].z, kx[3 * pair].w), 1);
                    bring_keys(codes_next, 3 * pair);
                    scores(2 * pair, codes_to_16<DT>(kx[3 * pair + 1].x, kx[3 * pair + 1].y), 2);
                    scores(2 * pair + 1, codes_to_16<DT>(kx[3 * pair + 1].z, kx[3 * pair + 1].w), 2);
                    bring_keys(codes_next, 3 * pair + 1);
                    scores(2 * pair + 1, codes_to_16<DT>(kx[3 * pair + 2].x, kx[3 * pair + 2].y), 0);
                    scores(2 * pair + 1, codes_to_16<DT>(kx[3 * pair + 2].z, kx[3 * pair + 2].w), 1);
                    bring_keys(codes_next, 3 * pair + 2);
                }
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
#pragma unroll
                    for (int c = 0; c < DP / 64; ++c) {
                        const int n = t * (DP / 64) + c;
                        const uint4 k0 = codes_to_16<DT>(kx[n].x, kx[n].y), k1 = codes_to_16<DT>(kx[n].z, kx[n].w);
                        scores(t, k0, 2 * c);
                        scores(t, k1, 2 * c + 1);
                    }
#pragma unroll
                    for (int c = 0; c < DP / 64; ++c) bring_keys(codes_next, t * (DP / 64) + c);
                }
            }

            if (here) {
                float to_log2 = score_factor(a, scales.x);
                const int from = (BLOCKS == kShared ? block & 0xffff : block) * kBlock;
                const bool partly = from + kBlock - 1 > last_least;
                const uint32_t have = (uint32_t)block >> 16;            // (kShared) the tokens that have the block
                const bool mine = BLOCKS != kShared || (have >> token & 1u), all = BLOCKS != kShared || have == tokens;
                const int scale_v = exponent_of(scales.y), unit_new = unit.with(scale_v);
                if (__builtin_expect(unit_new != unit.e, 0)) {
                    const float factor = pow2_held(unit.e - unit_new);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) o[mt][t] *= factor;
                    unit.e = unit_new;
                }
                const bool far = RunningUnit::far(scale_v, unit.e);
                const float to_unit = far ? 1.f : pow2_held(scale_v - unit.e);
                if (partly) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        const int left = last[mt] - from - 4 * quarter;     // scores i of tile t with 16 t + i <= left are seen
#pragma unroll
                        for (int t = 0; t < 4; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) z[mt][t][i] = 16 * t + i <= left ? z[mt][t][i] * to_log2 : -__builtin_inff();
                    }
                    to_log2 = 1.f;      // (a factor of zero would make NaN of what is masked)
                }
                uint4 p[MT][2];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    float most = z[mt][0][0];
#pragma unroll
                    for (int i = 1; i < 16; ++i) most = fmaxf(most, z[mt][i >> 2][i & 3]);
                    most = max_over_16(max_over_32(most)) * to_log2;
                    if (BLOCKS == kShared) most = mine ? most : -__builtin_inff();
                    if (__builtin_expect(__any(most - m[mt] > kSlack), 0)) {
                        const float m_new = fmaxf(m[mt], most - kLead);
                        const float factor = m_new == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m[mt] - m_new);
                        m[mt] = m_new;
                        l[mt] *= factor;
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) o[mt][t] *= factor;
                    }
                    const float base = m[mt] == -__builtin_inff() ? 0.f : -m[mt];
                    uint32_t w[8];
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[mt][i >> 2][i & 3], to_log2, base));
                        const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[mt][i >> 2][(i & 3) + 1], to_log2, base));
                        sum += e0;
                        sum += e1;
                        w[i >> 1] = pack2<FC_F16>(e0, e1);
                    }
                    if (BLOCKS == kShared && !all) {
                        sum = mine ? sum : 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = mine ? w[i] : 0;
                    }
                    l[mt] += sum;
                    p[mt][0] = make_uint4(w[0], w[1], w[2], w[3]);
                    p[mt][1] = make_uint4(w[4], w[5], w[6], w[7]);
                }

                if (__builtin_expect((partly || !all) && scales.y < 0.f, 0)) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        const int left = mine ? last[mt] - from - 4 * quarter : -1;
                        uint4 seen[2];
                        seen[0] = make_uint4(seen_pair(0, left), seen_pair(2, left), seen_pair(16, left), seen_pair(18, left));
                        seen[1] = make_uint4(seen_pair(32, left), seen_pair(34, left), seen_pair(48, left), seen_pair(50, left));
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            f32x4_t count = {0.f, 0.f, 0.f, 0.f};
                            count = mfma16<FC_F16>(nan_marks(vx[t].x, vx[t].y), seen[0], count);
                            count = mfma16<FC_F16>(nan_marks(vx[t].z, vx[t].w), seen[1], count);
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[mt][t][i] = count[i] > 0.f ? __builtin_nanf("") : o[mt][t][i];
                        }
                    }
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) vx[t] = without_nan(vx[t]);
                }
                if (__builtin_expect(far, 0)) {     // exact products in units of the block's scale, added to o in 32 bits; the weights below are zeros then
                    const float ratio = pow2_held(scale_v - unit.e);
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        __builtin_amdgcn_sched_barrier(0);      // (one after another, in few registers)
                        const uint4 v0 = codes_to_16<FC_F16>(vx[t].x, vx[t].y), v1 = codes_to_16<FC_F16>(vx[t].z, vx[t].w);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            f32x4_t adds = {0.f, 0.f, 0.f, 0.f};
                            adds = mfma16<FC_F16>(v0, p[mt][0], adds);
                            adds = mfma16<FC_F16>(v1, p[mt][1], adds);
                            o[mt][t] += adds * ratio;
                        }
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) p[mt][0] = p[mt][1] = make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    const uint4 v0 = codes_to_f16(vx[t].x, vx[t].y, to_unit), v1 = codes_to_f16(vx[t].z, vx[t].w, to_unit);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        o[mt][t] = mfma16<FC_F16>(v0, p[mt][0], o[mt][t]);
                        o[mt][t] = mfma16<FC_F16>(v1, p[mt][1], o[mt][t]);
                    }
                    bring_values(codes_next, t);
                }
            } else {
#pragma unroll
                for (int t = 0; t < kTiles; ++t) bring_values(codes_next, t);
            }
            block = block_next, pool = pool_next, scales = scales_next;
        }
    }
};

// sum over the four lanes that hold one row
__device__ __forceinline__ float row_sum(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// The number of blocks that a token with position `pos` has in its list.
__device__ __forceinline__ int listed_blocks(const AttnArgs &a, int pos) { return pos < 0 ? 0 : min(pos / kBlock + 1, a.selected_width); }

// Waves a SIMD that the registers allow without spilling.
template <int DP, int MT> constexpr int kOccupancy = DP * MT <= 64 ? 4 : DP * MT <= 128 ? 2 : 1;
constexpr int kListWaves = 4;

// Bound by memory where there are blocks enough: 64 tokens over caches of up to 8192, 8 heads of 128 with 4 queries each, 685 MB: 134 us, 5.1 TB/s, the rate of
// a large copy; one token over 131 000, 268 MB: 55 us, 4.9 TB/s.  Below, by round trips (lengths, table, scales and codes, pieces, join): one token over 1000: 8.5 us.
template <int DT, int DP, int MT, int WAVES, bool LIST> __global__ __launch_bounds__(64 * WAVES, (kOccupancy<DP, MT>)) void k_attend_rows(AttnArgs a)
{
    constexpr int kWaves = WAVES, kThreads = 64 * kWaves;
    constexpr int kTiles = DP / 16, kRows = 16 * MT, kPitch = DP + 4;
    extern __shared__ __align__(16) float lds[];
    float *const lds_o = lds, *const lds_m = lds + kWaves * kRows * kPitch, *const lds_l = lds_m + kWaves * kRows;
    int32_t *const lds_flag = reinterpret_cast<int32_t *>(lds_l + kWaves * kRows);
    const KvGeom &g = a.kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;

    uint32_t at = blockIdx.x;
    const int split = at % a.splits;
    at /= a.splits;
    const int64_t unit = at;
    const int tile = at % a.tiles;
    at /= a.tiles;
    const int h = at % g.kv_heads, b = at / g.kv_heads;
    const Sequence s = sequence_of(g, b);

    // the tile's rows: from head0 of new token token0 on (LIST: of this token only)
    int token0, head0, rows;
    if constexpr (LIST) {
        const int per_token = (a.group + kRows - 1) / kRows;
        token0 = tile / per_token;
        head0 = tile % per_token * kRows;
        rows = token0 < s.n ? min(a.group - head0, kRows) : 0;
    } else {
        const RowPlace p = row_place(a, tile * kRows);
        token0 = p.token, head0 = p.head;
        rows = min(max(s.n * a.group - tile * kRows, 0), kRows);
    }
    if (rows <= 0) return;
    const int token_last = LIST ? token0 : token0 + row_place(a, head0 + rows - 1).token;
    const int last_most = a.causal ? s.pos0 + token_last : s.len - 1;
    const int blocks = LIST ? listed_blocks(a, last_most) : last_most < 0 ? 0 : last_most / kBlock + 1;
    const int active = max((blocks + a.per_split - 1) / a.per_split, 1);
    if (split >= active) return;
    const int end = min(blocks, (split + 1) * a.per_split);

    Rows<DT, DP, MT> w;
    w.clear();
    w.last_least = a.causal ? s.pos0 + token0 : s.len - 1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        // (rows behind the last repeat it and are left out below)
        const int r = min(16 * mt + col, rows - 1);
        const RowPlace p = LIST ? RowPlace{0, head0 + r} : row_place(a, head0 + r);
        w.last[mt] = a.causal ? s.pos0 + token0 + p.token : s.len - 1;
        w.bring_queries(a, mt, a.q + (s.row0 + token0 + p.token) * a.q_row + (int64_t)(h * a.group + p.head) * a.q_head);
    }
    const int32_t *const list = LIST ? a.selected + ((int64_t)(s.row0 + token0) * g.kv_heads + h) * a.selected_width : nullptr;
    w.template run<LIST ? kListed : kAllBlocks>(a, b, h, list, split * a.per_split + wave, kWaves, end);

    // the waves' parts through LDS
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int r = wave * kRows + 16 * mt + col;
        const float sum = row_sum(w.l[mt]);
        if (quarter == 0) {
            lds_m[r] = w.m[mt];
            lds_l[r] = sum;
        }
        if (16 * mt + col < rows)
#pragma unroll
            for (int t = 0; t < kTiles; ++t) *reinterpret_cast<f32x4_t *>(lds_o + r * kPitch + 16 * t + 4 * quarter) = w.o[mt][t] * w.unit.to_sums();
    }
    __syncthreads();
    constexpr int kPieces = DP / 4;
    const Pieces<DP> pieces(a, unit, kRows);
    auto out_row = [&](int r) {
        const RowPlace p = LIST ? RowPlace{0, head0 + r} : row_place(a, head0 + r);
        return (int64_t)(s.row0 + token0 + p.token) * a.heads + h * a.group + p.head;
    };
    for (int i = threadIdx.x; i < rows * kPieces; i += kThreads) {
        const int r = i / kPieces, c = i % kPieces * 4;
        float most = -__builtin_inff();
#pragma unroll
        for (int v = 0; v < kWaves; ++v) most = fmaxf(most, lds_m[v * kRows + r]);
        const float base = most == -__builtin_inff() ? 0.f : most;
        f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
        float total = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            const float f = __builtin_amdgcn_exp2f(lds_m[v * kRows + r] - base);
            total += f * lds_l[v * kRows + r];
            sum += f * *reinterpret_cast<const f32x4_t *>(lds_o + (v * kRows + r) * kPitch + c);
        }
        if (active == 1) {
            finish_row<DT>(a, out_row(r), c, sum, most, total);
        } else {
            pieces.put((uint32_t)(split * kRows * kPieces + i), sum);
            if (c == 0) pieces.put_ml((uint32_t)(split * kRows + r), most, total);
        }
    }
    if (active == 1 || !last_to_arrive(a, unit, active, lds_flag)) return;
    auto place = [](int item) { return ItemPlace{item / kPieces, item % kPieces * 4}; };
    join_pieces<DT, DP, kThreads>(a, pieces, rows * kPieces, kRows, active, lds, place, out_row);
}

// Bound by the vector unit, which converts a block's codes for the few rows of one token, and by latency where there are few lists: 2294 lists of nine blocks,
// two heads of 96 with five queries each: 23.5 us, one round of waves.
// A wave takes up to 16 heads of one token and the token's whole list.  An XCD takes an eighth of the units in one piece: neighbouring tokens of a head
// share blocks.
template <int DT, int DP> __global__ __launch_bounds__(64 * kListWaves, (kOccupancy<DP, 1>)) void k_attend_lists(AttnArgs a)
{
    constexpr int kTiles = DP / 16;
    const KvGeom &g = a.kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;
    const uint32_t eighth = gridDim.x / 8;      // (the grid is a multiple of eight)
    uint32_t at = (blockIdx.x % 8 * eighth + blockIdx.x / 8) * kListWaves + wave;
    const int tile = at % a.tiles;
    at /= a.tiles;
    const int h = at % g.kv_heads, b = at / g.kv_heads;
    if (b >= g.batch) return;
    const Sequence s = sequence_of(g, b);
    const int per_token = (a.group + 15) / 16, token = tile / per_token, head0 = tile % per_token * 16;
    if (token >= s.n) return;
    const bool valid = head0 + col < a.group;
    const int pos = s.pos0 + token, head = min(head0 + col, a.group - 1);
    Rows<DT, DP, 1> w;
    w.clear();
    w.last_least = w.last[0] = pos;
    w.bring_queries(a, 0, a.q + (s.row0 + token) * a.q_row + (int64_t)(h * a.group + head) * a.q_head);
    w.template run<kListed>(a, b, h, a.selected + ((int64_t)(s.row0 + token) * g.kv_heads + h) * a.selected_width, 0, 1, listed_blocks(a, pos));
    const float sum = row_sum(w.l[0]);
    if (!valid) return;
    const int64_t row = (int64_t)(s.row0 + token) * a.heads + h * a.group + head;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) finish_row<DT>(a, row, 16 * t + 4 * quarter, w.o[0][t] * w.unit.to_sums(), w.m[0], sum);
}

// Bound by the vector unit as the lists alone are: 246 instructions a block beside the 32 matrix ones, most of them conversions of codes.  4096 tokens over 512 blocks, lists of 16,
// 8 heads of 128 with 4 queries each: 341 - 361 us (lists one a wave: 500).
// A wave takes a.shared neighbouring tokens of a sequence (a.shared * group <= 16 rows).  Their lists are put together in LDS: a mask of tokens for every block
// of the sequence, and the blocks with one, in order.  Blocks that neighbours share, the first and the last ones among them, are read and multiplied once,
// and the rows of the matrix instructions, of which one token fills `group`, are used.
template <int DT, int DP> __global__ __launch_bounds__(64 * kListWaves, (kOccupancy<DP, 1>)) void k_attend_shared(AttnArgs a)
{
    constexpr int kTiles = DP / 16;
    extern __shared__ __align__(16) uint32_t lds_words[];
    const KvGeom &g = a.kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4;
    const uint32_t eighth = gridDim.x / 8;      // (the grid is a multiple of eight)
    uint32_t at = (blockIdx.x % 8 * eighth + blockIdx.x / 8) * kListWaves + wave;
    const int tile = at % a.tiles;
    at /= a.tiles;
    const int h = at % g.kv_heads, b = at / g.kv_heads;
    if (b >= g.batch) return;
    const Sequence s = sequence_of(g, b);
    const int token0 = tile * a.shared, tokens = min(a.shared, s.n - token0);
    if (tokens <= 0) return;
    uint32_t *const words = lds_words + wave * (a.mask_words + a.entries);      // two blocks' masks a word
    int32_t *const entries = reinterpret_cast<int32_t *>(words + a.mask_words);

    const int pos = s.pos0 + token0, pos_last = pos + tokens - 1, blocks = pos_last < 0 ? 0 : pos_last / kBlock + 1;
    for (int i = lane; i < (blocks + 1) / 2; i += 64) words[i] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int32_t *const lists = a.selected + ((int64_t)(s.row0 + token0) * g.kv_heads + h) * a.selected_width;
    for (int i = lane; i < tokens * a.selected_width; i += 64) {
        const int t = i / a.selected_width;
        const int32_t block = lists[(int64_t)t * g.kv_heads * a.selected_width + i % a.selected_width];
        if ((uint32_t)block < (uint32_t)blocks) atomicOr(&words[block >> 1], 1u << (t + 16 * (block & 1)));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int count = 0;
    const uint64_t below = (1ull << lane) - 1;
    for (int i = 0; i < blocks; i += 64) {
        const int block = i + lane;
        const uint32_t have = block < blocks ? words[block >> 1] >> (16 * (block & 1)) & 0xffffu : 0;
        const uint64_t takes = __ballot(have != 0);
        if (have) entries[count + (int)__popcll(takes & below)] = block | (int32_t)(have << 16);
        count += (int)__popcll(takes);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");

    const int rows = tokens * a.group;
    const bool valid = col < rows;
    const RowPlace p = row_place(a, min(col, rows - 1));        // (rows behind the last repeat it and are left out below)
    Rows<DT, DP, 1> w;
    w.clear();
    w.last_least = pos;
    w.last[0] = pos + p.token;
    w.token = (uint32_t)p.token;
    w.tokens = (1u << tokens) - 1u;
    w.bring_queries(a, 0, a.q + (s.row0 + token0 + p.token) * a.q_row + (int64_t)(h * a.group + p.head) * a.q_head);
    w.template run<kShared>(a, b, h, entries, 0, 1, count);
    const float sum = row_sum(w.l[0]);
    if (!valid) return;
    const int64_t row = (int64_t)(s.row0 + token0 + p.token) * a.heads + h * a.group + p.head;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) finish_row<DT>(a, row, 16 * t + 4 * quarter, w.o[0][t] * w.unit.to_sums(), w.m[0], sum);
}

template <int DT, int DP, int MT, int WAVES, bool LIST> hipError_t run_rows(const AttnArgs &a, hipStream_t s)
{
    constexpr size_t lds = ((size_t)WAVES * 16 * MT * (DP + 4 + 2) + 4) * sizeof(float);
    if (lds > 64 * 1024) {
        const hipError_t e = raise_lds<k_attend_rows<DT, DP, MT, WAVES, LIST>>(lds);
        if (e != hipSuccess) return e;
    }
    const int64_t units = (int64_t)a.kv.batch * a.kv.kv_heads * a.tiles;
    k_attend_rows<DT, DP, MT, WAVES, LIST><<<dim3((uint32_t)(units * a.splits)), 64 * WAVES, lds, s>>>(a);
    return hipGetLastError();
}

template <int DT, int DP> hipError_t run_lists(const AttnArgs &a, bool whole, hipStream_t s)
{
    if (!whole) return run_rows<DT, DP, 1, 4, true>(a, s);
    if (a.shared > 1) {
        const size_t lds = (size_t)kListWaves * (a.mask_words + a.entries) * sizeof(uint32_t);
        const hipError_t e = raise_lds<k_attend_shared<DT, DP>>((size_t)kListWaves * kSharedMaxWords * sizeof(uint32_t));
        if (e != hipSuccess) return e;
        const int64_t waves = (int64_t)a.kv.batch * a.kv.kv_heads * a.tiles;
        k_attend_shared<DT, DP><<<dim3((uint32_t)((waves + 8 * kListWaves - 1) / (8 * kListWaves) * 8)), 64 * kListWaves, lds, s>>>(a);
        return hipGetLastError();
    }
    const int64_t units = (int64_t)a.kv.batch * a.kv.kv_heads * a.tiles;
    k_attend_lists<DT, DP><<<dim3((uint32_t)((units + 8 * kListWaves - 1) / (8 * kListWaves) * 8)), 64 * kListWaves, 0, s>>>(a);
    return hipGetLastError();
}

template <int DT, int DP> hipError_t run_dim(const AttnArgs &a, int rows_tile, int waves, hipStream_t s)
{
    if constexpr (DP <= 128) {
        if (rows_tile == 32) return run_rows<DT, DP, 2, 4, false>(a, s);
        if (waves == 8) return run_rows<DT, DP, 1, 8, false>(a, s);
    }
    return run_rows<DT, DP, 1, 4, false>(a, s);
}

} // namespace

hipError_t launch_attend_rows(const AttnArgs &a, int dtype, int rows_tile, int waves, hipStream_t s)
{
    const bool b = dtype == FC_BF16;
    switch (a.kv.dp) {
    case 64: return b ? run_dim<FC_BF16, 64>(a, rows_tile, waves, s) : run_dim<FC_F16, 64>(a, rows_tile, waves, s);
    case 96: return b ? run_dim<FC_BF16, 96>(a, rows_tile, waves, s) : run_dim<FC_F16, 96>(a, rows_tile, waves, s);
    case 128: return b ? run_dim<FC_BF16, 128>(a, rows_tile, waves, s) : run_dim<FC_F16, 128>(a, rows_tile, waves, s);
    case 192: return b ? run_dim<FC_BF16, 192>(a, rows_tile, waves, s) : run_dim<FC_F16, 192>(a, rows_tile, waves, s);
    default: return b ? run_dim<FC_BF16, 256>(a, rows_tile, waves, s) : run_dim<FC_F16, 256>(a, rows_tile, waves, s);
    }
}

hipError_t launch_attend_lists(const AttnArgs &a, int dtype, bool whole, hipStream_t s)
{
    const bool b = dtype == FC_BF16;
    switch (a.kv.dp) {
    case 64: return b ? run_lists<FC_BF16, 64>(a, whole, s) : run_lists<FC_F16, 64>(a, whole, s);
    case 96: return b ? run_lists<FC_BF16, 96>(a, whole, s) : run_lists<FC_F16, 96>(a, whole, s);
    case 128: return b ? run_lists<FC_BF16, 128>(a, whole, s) : run_lists<FC_F16, 128>(a, whole, s);
    case 192: return b ? run_lists<FC_BF16, 192>(a, whole, s) : run_lists<FC_F16, 192>(a, whole, s);
    default: return b ? run_lists<FC_BF16, 256>(a, whole, s) : run_lists<FC_F16, 256>(a, whole, s);
    }
}

} // namespace fc
